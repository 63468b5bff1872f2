// New tokens into the paged cache: q and k normed per head (optional) and
// rotated, k and v written to their pages, q to q_out, in one launch.
//
// The token at position p turns pair j of its first rot_dim values by the
// angle p inv_freq[j].  The product is formed in fp64 (exact below position 2^29,
// a factor of 24 bits and one of 29) and reduced to a part of a turn there, off
// by 2^-51 of itself at most, so the angle is as good at position 10^6 as at 1;
// sine and cosine are fp32.  Everything else is computed in fp32 and rounded
// once.
//
// A group of LG lanes owns a head vector, a lane 4 pairs: values 4c.. and
// rot_dim/2 + 4c.. (half layout) or 8c..8c+7 (interleaved, and the part that
// is not rotated), so a pair never leaves its lane and one sine serves every
// head that the lane's group visits.
//
// Bound by memory: 8593 tokens of 32 + 8 + 8 heads of 128, with per-head norms,
// 211 MB read and written in 51 to 52.5 us, 4.0 to 4.1 TB/s (36 us without norms
// where the buffers stay in the last cache); a few tokens by the chain length ->
// page -> store, 3 us.

#include <math.h>

#include "../../include/cl.h"
#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

struct Raw {                   // four 16-bit values as they stand
    uint32_t a, b;
};

struct Quad {
    float v[4];
};

// A lane's two quads at `lo` and `hi`: neighbours (hi = lo + 4, 16-byte aligned)
// in one access.
template <bool VEC>
__device__ __forceinline__ void load8(const uint16_t* p, int lo, int hi, bool apart, Raw& x, Raw& y) {
    if constexpr (VEC) {
        if (apart) {
            const u32x2 u = *reinterpret_cast<const u32x2*>(p + lo), v = *reinterpret_cast<const u32x2*>(p + hi);
            x = Raw{u[0], u[1]};
            y = Raw{v[0], v[1]};
        } else {
            const u32x4 u = *reinterpret_cast<const u32x4*>(p + lo);
            x = Raw{u[0], u[1]};
            y = Raw{u[2], u[3]};
        }
    } else {
        const auto two = [](const uint16_t* q) { return q[0] | static_cast<uint32_t>(q[1]) << 16; };
        x = Raw{two(p + lo), two(p + lo + 2)};
        y = Raw{two(p + hi), two(p + hi + 2)};
    }
}

// STREAM: a prompt's results (four heads a group, see choose) are stored past the
// L2 caches (8593 tokens 56.5 -> 47.3 us when it was changed).
// Attention behind the call is no slower for it: 1500 tokens, both, 56.2 us
// against 57.2 with ordinary stores, 3000 103.5 / 104.8, 8593 627 / 626.
template <bool STREAM, class T>
__device__ __forceinline__ void put(uint16_t* p, T v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<T*>(p));
    else *reinterpret_cast<T*>(p) = v;
}

template <bool VEC, bool STREAM>
__device__ __forceinline__ void store8(uint16_t* p, int lo, int hi, bool apart, Raw x, Raw y) {
    if constexpr (VEC) {
        if (apart) {
            put<STREAM>(p + lo, u32x2{x.a, x.b});
            put<STREAM>(p + hi, u32x2{y.a, y.b});
        } else {
            put<STREAM>(p + lo, u32x4{x.a, x.b, y.a, y.b});
        }
    } else {
        const auto two = [](uint16_t* q, uint32_t v) {
            q[0] = static_cast<uint16_t>(v);
            q[1] = static_cast<uint16_t>(v >> 16);
        };
        two(p + lo, x.a), two(p + lo + 2, x.b);
        two(p + hi, y.a), two(p + hi + 2, y.b);
    }
}

__device__ __forceinline__ Quad widen(Raw r, int dt) {
    return Quad{{act_to_f32(static_cast<uint16_t>(r.a & 0xffff), dt), act_to_f32(static_cast<uint16_t>(r.a >> 16), dt),
                 act_to_f32(static_cast<uint16_t>(r.b & 0xffff), dt), act_to_f32(static_cast<uint16_t>(r.b >> 16), dt)}};
}

__device__ __forceinline__ Raw narrow(const Quad& q, int dt) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = dt == DT_FP16 ? f32_to_f16_bits(q.v[i]) : f32_to_bf16_bits(q.v[i]);
    return Raw{b[0] | b[1] << 16, b[2] | b[3] << 16};
}

// Heads of a token in the order q, k, v; group `first` takes every
// step-th head, HP of them at most: their loads are issued together, ahead of
// the chain that finds the token's page.  head_dim and rot_dim are multiples
// of 8 (LG lanes of 8 values cover a head).
template <int LG, bool VEC, int HP>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a, int step) {
    const int t = static_cast<int>(a.first + blockIdx.x);
    const int lane = threadIdx.x % LG;
    const int first = blockIdx.y * (blockDim.x / LG) + threadIdx.x / LG;
    const int D = a.cache.dim, dt = a.cache.dtype;
    const int Hq = a.q ? a.q_heads : 0, Hk = a.cache.heads;

    const int at = 8 * lane;                          // first of the lane's 8 values in memory order
    const bool live = at < D;
    const bool turned = a.rope.inv_freq && at < a.rope.rot_dim;
    const bool half = turned && !a.rope.interleaved;
    const int lo = half ? 4 * lane : at, hi = half ? a.rope.rot_dim / 2 + 4 * lane : at + 4;

    Raw x[HP], y[HP];
#pragma unroll
    for (int i = 0; i < HP; ++i) {
        const int h = first + i * step;
        if (!live || h >= Hq + 2 * Hk) continue;
        const bool is_v = h >= Hq + Hk;
        const uint16_t* src = h < Hq ? a.q + static_cast<long long>(t) * a.q_stride + static_cast<size_t>(h) * D
                              : is_v ? a.v + static_cast<long long>(t) * a.v_stride + static_cast<size_t>(h - Hq - Hk) * D
                                     : a.k + static_cast<long long>(t) * a.k_stride + static_cast<size_t>(h - Hq) * D;
        load8<VEC>(src, is_v ? at : lo, is_v ? at + 4 : hi, half && !is_v, x[i], y[i]);
    }

    // the token's place: the same for the whole workgroup
    const int s = seq_of(a.batch, t);
    int pos = 0, page = -1, row = 0;
    bool owned = false;                               // the token is some sequence's
    if (s >= 0) {
        const Seq q = load_seq(a.batch, s);
        if (t < q.start + q.count) {
            owned = true;
            pos = q.keys - q.count + (t - q.start);
            const int mine = pos - a.batch.prefix_len;
            if (mine >= 0) {
                page = a.batch.page_table[static_cast<size_t>(s) * a.batch.table_width + (mine >> a.cache.page_shift)];
                row = mine & ((1 << a.cache.page_shift) - 1);
            }
        }
    }
    const bool stored = page >= 0 && page < a.cache.num_pages;
    const int angle_pos = a.positions ? a.positions[t] : pos;
    float cs[4], sn[4];
    if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double turns = static_cast<double>(angle_pos) * static_cast<double>(a.rope.inv_freq[4 * lane + i]) *
                                 0.15915494309189533577;         // 1 / (2 pi)
            sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sn[i], &cs[i]);
            sn[i] *= a.rope.magnitude;
            cs[i] *= a.rope.magnitude;
        }
    }

#pragma unroll
    for (int n = 0; n < HP; ++n) {
        const int h = first + n * step;
        if (h >= Hq + 2 * Hk) continue;
        const bool is_q = h < Hq, is_v = h >= Hq + Hk;
        const int head = is_q ? h : is_v ? h - Hq - Hk : h - Hq;
        uint16_t* dst;
        if (is_q) {
            dst = a.q_out + (static_cast<size_t>(t) * Hq + head) * D;
        } else {
            const size_t slot = ((static_cast<size_t>(stored ? page : 0) * Hk + head) << a.cache.page_shift) + row;
            dst = (is_v ? a.cache.v : a.cache.k) + slot * D;
        }
        if (is_v) {
            if (live && stored) {
                store8<VEC, (HP > 1)>(dst, at, at + 4, false, x[n], y[n]);
            }
            continue;
        }
        Quad u = live ? widen(x[n], dt) : Quad{}, v = live ? widen(y[n], dt) : Quad{};
        const uint16_t* w = is_q ? a.q_norm : a.k_norm;
        if (w) {
            float s2 = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) s2 += u.v[i] * u.v[i] + v.v[i] * v.v[i];
#pragma unroll
            for (int off = LG / 2; off > 0; off >>= 1) s2 += __shfl_xor(s2, off, 64);
            const float r = 1.0f / sqrtf(s2 / static_cast<float>(D) + a.eps);
            if (live) {
                Raw rx, ry;
                load8<VEC>(w, lo, hi, half, rx, ry);
                const Quad wx = widen(rx, dt), wy = widen(ry, dt);
#pragma unroll
                for (int i = 0; i < 4; ++i) u.v[i] *= r * wx.v[i], v.v[i] *= r * wy.v[i];
            }
        }
        if (half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = u.v[i], q = v.v[i];
                u.v[i] = p * cs[i] - q * sn[i];
                v.v[i] = p * sn[i] + q * cs[i];
            }
        } else if (turned) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                float p = u.v[i], q = u.v[i + 1];
                u.v[i] = p * cs[i / 2] - q * sn[i / 2];
                u.v[i + 1] = p * sn[i / 2] + q * cs[i / 2];
                p = v.v[i], q = v.v[i + 1];
                v.v[i] = p * cs[2 + i / 2] - q * sn[2 + i / 2];
                v.v[i + 1] = p * sn[2 + i / 2] + q * cs[2 + i / 2];
            }
        }
        if (live && (is_q ? owned : stored)) {
            store8<VEC, (HP > 1)>(dst, lo, hi, half, narrow(u, dt), narrow(v, dt));
        }
    }
}

template <int LG, int HP>
hipError_t launch(AppendArgs a, bool vec, int blocks, hipStream_t st) {
    const int step = blocks * (256 / LG);
    return launch_all(a.batch.tokens, [&](unsigned first, unsigned count) {
        a.first = first;
        const dim3 grid(count, blocks);
        if (vec) hipLaunchKernelGGL((kv_append_kernel<LG, true, HP>), grid, dim3(256), 0, st, a, step);
        else hipLaunchKernelGGL((kv_append_kernel<LG, false, HP>), grid, dim3(256), 0, st, a, step);
    });
}

// A lane group takes one head where workgroups are few (latency) and up to
// four of a token's where they are many, which share its sines and its page.
template <int LG>
hipError_t choose(const AppendArgs& a, bool vec, hipStream_t st) {
    constexpr int per = 256 / LG;
    const int heads = (a.q ? a.q_heads : 0) + 2 * a.cache.heads;
    const int blocks = (heads + per - 1) / per;
    if (static_cast<long long>(a.batch.tokens) * blocks < 2048) return launch<LG, 1>(a, vec, blocks, st);
    return launch<LG, 4>(a, vec, (heads + 4 * per - 1) / (4 * per), st);
}

bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

void rope_frequencies(int rot_dim, double base, int kind, double factor, double trained_len, double low, double high,
                      float* inv_freq, float* magnitude) {
    const double two_pi = 6.283185307179586477;
    if (kind == CL_ROPE_BASE && rot_dim > 2) base *= pow(factor, rot_dim / (rot_dim - 2.0));
    // the pair that makes t turns over the trained length
    const auto pair_of = [&](double t) { return rot_dim * log(trained_len / (two_pi * t)) / (2.0 * log(base)); };
    double first = 0.0, last = 1.0;
    if (kind == CL_ROPE_RAMP) {
        first = fmax(floor(pair_of(high)), 0.0);
        last = fmin(ceil(pair_of(low)), rot_dim - 1.0);
        if (last <= first) last = first + 0.001;
    }
    for (int j = 0; j < rot_dim / 2; ++j) {
        const double f = pow(base, -2.0 * j / rot_dim);
        double kept = 1.0;                            // weight of the unscaled frequency
        if (kind == CL_ROPE_LINEAR) kept = 0.0;
        if (kind == CL_ROPE_BANDS) kept = (trained_len * f / two_pi - low) / (high - low);
        if (kind == CL_ROPE_RAMP) kept = 1.0 - (j - first) / (last - first);
        kept = fmin(fmax(kept, 0.0), 1.0);
        const double scaled = kind == CL_ROPE_PLAIN || kind == CL_ROPE_BASE ? f : f / factor;
        inv_freq[j] = static_cast<float>(kept * f + (1.0 - kept) * scaled);
    }
    *magnitude = kind == CL_ROPE_RAMP ? static_cast<float>(0.1 * log(factor) + 1.0) : 1.0f;
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st) {
    const bool vec = wide(a.q) && wide(a.k) && wide(a.v) && wide(a.q_out) && wide(a.q_norm) && wide(a.k_norm) &&
                     a.q_stride % 8 == 0 && a.k_stride % 8 == 0 && a.v_stride % 8 == 0;
    if (a.cache.dim <= 64) return choose<8>(a, vec, st);
    if (a.cache.dim <= 128) return choose<16>(a, vec, st);
    return choose<32>(a, vec, st);
}

}  // namespace cl
