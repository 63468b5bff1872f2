// New tokens into the paged cache: q and k normed per head (optional) and
// rotated, k and v written to their pages, q to q_out, in one launch.
//
// The token at position p turns pair j of its first rot_dim values by the
// angle p inv_freq[j].  The product is formed in fp64 (exact: 24 by 31 bits)
// and reduced to a part of a turn there, so the angle is as exact at position
// 10^6 as at 1; sine and cosine are fp32.  Everything is computed in fp32 and
// rounded once.
//
// A group of LG lanes owns a head vector, a lane 4 pairs: values 4c.. and
// rot_dim/2 + 4c.. (half layout) or 8c..8c+7 (interleaved, and the part that
// is not rotated), so a pair never leaves its lane and one sine serves every
// head that the lane's group visits.

#include <math.h>

#include "../../include/cl.h"
#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

struct Quad {
    float v[4];
};

template <bool VEC>
__device__ __forceinline__ Quad load4(const uint16_t* p, int at, int dt) {
    Quad q;
    if constexpr (VEC) {
        const u32x2 u = *reinterpret_cast<const u32x2*>(p + at);
        const uint32_t a = u[0], b = u[1];
        q.v[0] = act_to_f32(static_cast<uint16_t>(a & 0xffff), dt);
        q.v[1] = act_to_f32(static_cast<uint16_t>(a >> 16), dt);
        q.v[2] = act_to_f32(static_cast<uint16_t>(b & 0xffff), dt);
        q.v[3] = act_to_f32(static_cast<uint16_t>(b >> 16), dt);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) q.v[i] = act_to_f32(p[at + i], dt);
    }
    return q;
}

__device__ __forceinline__ uint32_t round_bits(float v, int dt) {
    return dt == DT_FP16 ? f32_to_f16_bits(v) : f32_to_bf16_bits(v);
}

template <bool VEC>
__device__ __forceinline__ void store4(uint16_t* p, int at, int dt, const Quad& q) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = round_bits(q.v[i], dt);
    if constexpr (VEC) {
        *reinterpret_cast<u32x2*>(p + at) = u32x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[at + i] = static_cast<uint16_t>(b[i]);
    }
}

// Heads of a token in the order q, k, v; group `first` of `step` groups takes
// every step-th head.  head_dim is a multiple of 8 and rot_dim of 8 (LG lanes
// of 8 values cover a head).
template <int LG, bool VEC>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a, int groups_per_token) {
    const int t = blockIdx.x;
    const int lane = threadIdx.x % LG;
    const int first = blockIdx.y * (blockDim.x / LG) + threadIdx.x / LG;
    const int D = a.cache.dim, dt = a.cache.dtype;

    // the token's place: the same for the whole workgroup
    const int s = seq_of(a.batch, t);
    int pos = 0, page = -1, row = 0;
    if (s >= 0) {
        const Seq q = load_seq(a.batch, s);
        if (t < q.start + q.count) {
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

    const int at = 8 * lane;                          // first of the lane's 8 values in memory order
    const bool live = at < D;
    const bool turned = a.rope.inv_freq && at < a.rope.rot_dim;
    const bool half = turned && !a.rope.interleaved;
    const int lo = half ? 4 * lane : at, hi = half ? a.rope.rot_dim / 2 + 4 * lane : at + 4;
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

    const int Hq = a.q ? a.q_heads : 0, Hk = a.cache.heads;
    for (int h = first; h < Hq + 2 * Hk; h += groups_per_token) {
        const bool is_q = h < Hq, is_v = h >= Hq + Hk;
        const int head = is_q ? h : is_v ? h - Hq - Hk : h - Hq;
        const uint16_t* src = is_q   ? a.q + static_cast<long long>(t) * a.q_stride
                              : is_v ? a.v + static_cast<long long>(t) * a.v_stride
                                     : a.k + static_cast<long long>(t) * a.k_stride;
        src += static_cast<size_t>(head) * D;
        uint16_t* dst;
        if (is_q) {
            dst = a.q_out + (static_cast<size_t>(t) * Hq + head) * D;
        } else {
            const size_t slot = ((static_cast<size_t>(stored ? page : 0) * Hk + head) << a.cache.page_shift) + row;
            dst = (is_v ? a.cache.v : a.cache.k) + slot * D;
        }
        if (is_v) {
            if (live && stored) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if constexpr (VEC)
                        *reinterpret_cast<u32x2*>(dst + at + 4 * c) = *reinterpret_cast<const u32x2*>(src + at + 4 * c);
                    else
                        for (int i = 0; i < 4; ++i) dst[at + 4 * c + i] = src[at + 4 * c + i];
                }
            }
            continue;
        }
        Quad x{}, y{};
        if (live) {
            x = load4<VEC>(src, lo, dt);
            y = load4<VEC>(src, hi, dt);
        }
        const uint16_t* w = is_q ? a.q_norm : a.k_norm;
        if (w) {
            float s2 = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) s2 += x.v[i] * x.v[i] + y.v[i] * y.v[i];
#pragma unroll
            for (int off = LG / 2; off > 0; off >>= 1) s2 += __shfl_xor(s2, off, 64);
            const float r = 1.0f / sqrtf(s2 / static_cast<float>(D) + a.eps);
            if (live) {
                const Quad wx = load4<VEC>(w, lo, dt), wy = load4<VEC>(w, hi, dt);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[i] *= r * wx.v[i], y.v[i] *= r * wy.v[i];
            }
        }
        if (half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = x.v[i], v = y.v[i];
                x.v[i] = u * cs[i] - v * sn[i];
                y.v[i] = u * sn[i] + v * cs[i];
            }
        } else if (turned) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                float u = x.v[i], v = x.v[i + 1];
                x.v[i] = u * cs[i / 2] - v * sn[i / 2];
                x.v[i + 1] = u * sn[i / 2] + v * cs[i / 2];
                u = y.v[i], v = y.v[i + 1];
                y.v[i] = u * cs[2 + i / 2] - v * sn[2 + i / 2];
                y.v[i + 1] = u * sn[2 + i / 2] + v * cs[2 + i / 2];
            }
        }
        if (live && (is_q || stored)) {
            store4<VEC>(dst, lo, dt, x);
            store4<VEC>(dst, hi, dt, y);
        }
    }
}

template <int LG>
hipError_t launch(const AppendArgs& a, bool vec, hipStream_t st) {
    const int heads = (a.q ? a.q_heads : 0) + 2 * a.cache.heads;
    constexpr int per = 256 / LG;
    const int blocks = (heads + per - 1) / per;
    const dim3 grid(a.batch.tokens, blocks);
    if (vec)
        hipLaunchKernelGGL((kv_append_kernel<LG, true>), grid, dim3(256), 0, st, a, blocks * per);
    else
        hipLaunchKernelGGL((kv_append_kernel<LG, false>), grid, dim3(256), 0, st, a, blocks * per);
    return hipGetLastError();
}

bool even8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

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
    const bool vec = even8(a.q) && even8(a.k) && even8(a.v) && even8(a.q_out) && even8(a.q_norm) && even8(a.k_norm) &&
                     a.q_stride % 4 == 0 && a.k_stride % 4 == 0 && a.v_stride % 4 == 0;
    if (a.cache.dim <= 64) return launch<8>(a, vec, st);
    if (a.cache.dim <= 128) return launch<16>(a, vec, st);
    return launch<32>(a, vec, st);
}

}  // namespace cl
