// New tokens into a cache of e4m3 codes, and rows of a cache back out.
//
// A block of rows of a head shares a power of two: value = code 2^(scale - 127).
// The exponent is the smallest e with max |x| <= 448 2^e over the block's rows,
// held in a range that keeps every decoded value finite and normal in the
// cache's type (in fp16, whole in its subnormals).  e4m3 is a floating-point type,
// so a power of two loses nothing against a finer scale: a value keeps its 4
// bits wherever it stands between the type's ends, and only where the smallest
// magnitudes run out (2^-9 against 448) depends on the scale.  It buys two things: a decoded value is
// exactly one of the 16-bit type, and a block whose maximum grows later is
// rescaled exactly, but for codes that move below 2^-6.
//
// The workgroups of the first new token of a block (its y part behind the
// queries') take the block's rows, a wave for K or V of one head: one pass finds
// the maximum, a second one forms the same values again and stores them.  Rows that stood in
// the block before keep its exponent as a lower bound, and are rescaled where it
// grows.  Values are computed in fp32 and rounded once, to the code.

#include <math.h>

#include "append_common.h"
#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The exponents' range of a type, and the largest magnitude that is held: larger
// ones (behind a rotation or a norm) become it.
__device__ __forceinline__ int exponent_low(int dt) { return dt == DT_FP16 ? -15 : -117; }
__device__ __forceinline__ int exponent_high(int dt) { return dt == DT_FP16 ? 8 : 120; }
__device__ __forceinline__ float held_most(int dt) { return dt == DT_FP16 ? 61440.f : 0x1.ep127f; }

__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, static_cast<uint32_t>(max(e, -126) + 127) << 23); }

// Four values to codes; an infinity or NaN is the code of NaN.
__device__ __forceinline__ uint32_t encode4(const Quad& q, float inverse, float most) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = fminf(fmaxf(q.v[i], -most), most) * inverse;
        x[i] = fabsf(q.v[i]) <= 3.4028234663852886e38f ? v : NAN;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    return static_cast<uint32_t>(w);
}

__device__ __forceinline__ uint32_t rescale4(uint32_t c, float f) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, w, true);
    return static_cast<uint32_t>(w);
}

// One head vector of a token in a group of LG lanes: its norm (w) and rotation.
template <int LG>
__device__ __forceinline__ void norm_and_turn(const AppendArgs& a, int angle_pos, const uint16_t* w, bool vec_w, int lane,
                                              bool live, int lo, int hi, bool half, bool turned, Quad& u, Quad& v) {
    const int dt = a.cache.dtype;
    if (w) {
        float s2 = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) s2 += u.v[i] * u.v[i] + v.v[i] * v.v[i];
#pragma unroll
        for (int off = LG / 2; off > 0; off >>= 1) s2 += __shfl_xor(s2, off, 64);
        const float r = 1.0f / sqrtf(s2 / static_cast<float>(a.cache.dim) + a.eps);
        if (live) {
            Raw rx, ry;
            if (vec_w) load8<true>(w, lo, hi, half, rx, ry);
            else load8<false>(w, lo, hi, half, rx, ry);
            const Quad wx = widen(rx, dt), wy = widen(ry, dt);
#pragma unroll
            for (int i = 0; i < 4; ++i) u.v[i] *= r * wx.v[i], v.v[i] *= r * wy.v[i];
        }
    }
    if (!turned) return;
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double turns = static_cast<double>(angle_pos) * static_cast<double>(a.rope.inv_freq[4 * lane + i]) *
                             0.15915494309189533577;         // 1 / (2 pi)
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sn[i], &cs[i]);
        sn[i] *= a.rope.magnitude;
        cs[i] *= a.rope.magnitude;
    }
    if (half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = u.v[i], q = v.v[i];
            u.v[i] = p * cs[i] - q * sn[i];
            v.v[i] = p * sn[i] + q * cs[i];
        }
    } else {
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
}

template <int LG, bool VEC>
__global__ __launch_bounds__(256) void kv_append8_kernel(AppendArgs a, int q_blocks) {
    constexpr int PER = 256 / LG, ROWS = 64 / LG;     // head vectors of a workgroup, of a wave
    const int t = static_cast<int>(a.first + blockIdx.x);
    const int lane = threadIdx.x % LG;
    const int D = a.cache.dim, dt = a.cache.dtype, Hk = a.cache.heads;
    const int at = 8 * lane;                          // first of the lane's 8 values in memory order
    const bool live = at < D;
    const bool rotary = a.rope.inv_freq && at < a.rope.rot_dim;
    const bool half = rotary && !a.rope.interleaved;
    const int lo = half ? 4 * lane : at, hi = half ? a.rope.rot_dim / 2 + 4 * lane : at + 4;

    const int s = seq_of(a.batch, t);
    if (s < 0) return;
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count) return;               // no sequence's row
    const int pos = q.keys - q.count + (t - q.start);

    if (static_cast<int>(blockIdx.y) < q_blocks) {
        const int h = blockIdx.y * PER + threadIdx.x / LG;
        if (h >= a.q_heads) return;                   // whole groups: nothing is exchanged between them
        Raw x = {}, y = {};
        if (live) load8<VEC>(a.q + static_cast<long long>(t) * a.q_stride + static_cast<size_t>(h) * D, lo, hi, half, x, y);
        Quad u = widen(x, dt), v = widen(y, dt);
        norm_and_turn<LG>(a, a.positions ? a.positions[t] : pos, a.q_norm, VEC, lane, live, lo, hi, half, rotary, u, v);
        if (live) store8<VEC, false>(a.q_out + (static_cast<size_t>(t) * a.q_heads + h) * D, lo, hi, half, narrow(u, dt), narrow(v, dt));
        return;
    }

    const int mine = pos - a.batch.prefix_len, block = 1 << a.cache.block_shift;
    const int before = mine & (block - 1);            // rows of the block that stood there
    if (mine < 0 || (before != 0 && t != q.start)) return;
    const int page = a.batch.page_table[static_cast<size_t>(s) * a.batch.table_width + (mine >> a.cache.page_shift)];
    if (page < 0 || page >= a.cache.num_pages) return;
    const int unit = 4 * (blockIdx.y - q_blocks) + threadIdx.x / 64;
    if (unit >= 2 * Hk) return;
    const bool is_v = unit >= Hk;
    const int head = is_v ? unit - Hk : unit;
    const int rows = min(block - before, q.start + q.count - t);
    const int first = ((page * Hk + head) << a.cache.page_shift) + (mine & ((1 << a.cache.page_shift) - 1));
    uint8_t* const scale = (is_v ? a.cache.v_scale : a.cache.k_scale) + (static_cast<unsigned>(first) >> a.cache.block_shift);
    uint8_t* const codes = reinterpret_cast<uint8_t*>(is_v ? a.cache.v : a.cache.k) + static_cast<size_t>(first) * D;
    const uint16_t* const src = (is_v ? a.v : a.k) + static_cast<size_t>(head) * D;
    const long long stride = is_v ? a.v_stride : a.k_stride;
    const int group = (threadIdx.x & 63) / LG;
    const bool turned = rotary && !is_v, apart = half && !is_v;
    const int l = is_v ? at : lo, r = is_v ? at + 4 : hi;

    const auto values = [&](int i, Quad& u, Quad& v) {            // of the block's i-th new row
        Raw x = {}, y = {};
        const bool there = live && i < rows;
        if (there) load8<VEC>(src + static_cast<long long>(t + i) * stride, l, r, apart, x, y);
        u = widen(x, dt), v = widen(y, dt);
        if (!is_v) {
            const int p = a.positions ? (i < rows ? a.positions[t + i] : 0) : pos + i;
            norm_and_turn<LG>(a, p, a.k_norm, VEC, lane, there, l, r, apart, turned, u, v);
        }
    };

    const float most = held_most(dt);
    float top = 0.f;
    for (int i = 0; i < rows; i += ROWS) {
        Quad u, v;
        values(i + group, u, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = fabsf(u.v[j]), y = fabsf(v.v[j]);
            top = fmaxf(top, x <= 3.4028234663852886e38f ? x : 0.f);
            top = fmaxf(top, y <= 3.4028234663852886e38f ? y : 0.f);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const uint32_t bits = __builtin_bit_cast(uint32_t, top);
    const int low = exponent_low(dt), high = exponent_high(dt);
    // 448 = 1.75 2^8
    int e = min(max(static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u), low), high);
    const int e0 = before ? min(max(static_cast<int>(*scale) - 127, low), high) : e;
    if (e0 >= e) {
        e = e0;
    } else {
        uint32_t* const old = reinterpret_cast<uint32_t*>(codes - static_cast<size_t>(before) * D);
        const float f = power_of_two(e0 - e);
        for (int i = threadIdx.x & 63; i < before * D / 4; i += 64) old[i] = rescale4(old[i], f);
    }
    if ((threadIdx.x & 63) == 0) *scale = static_cast<uint8_t>(e + 127);
    const float inverse = power_of_two(-e);
    for (int i = 0; i < rows; i += ROWS) {
        Quad u, v;
        values(i + group, u, v);
        if (!live || i + group >= rows) continue;
        uint8_t* const to = codes + static_cast<size_t>(i + group) * D;
        const uint32_t x = encode4(u, inverse, most), y = encode4(v, inverse, most);
        if (apart) {
            *reinterpret_cast<uint32_t*>(to + l) = x;
            *reinterpret_cast<uint32_t*>(to + r) = y;
        } else {
            *reinterpret_cast<u32x2*>(to + l) = u32x2{x, y};
        }
    }
}

template <int LG>
hipError_t launch(AppendArgs a, bool vec, hipStream_t st) {
    const int q_blocks = a.q ? (a.q_heads + 256 / LG - 1) / (256 / LG) : 0;
    return launch_all(a.batch.tokens, [&](unsigned first, unsigned count) {
        a.first = first;
        const dim3 grid(count, q_blocks + (2 * a.cache.heads + 3) / 4);
        if (vec) hipLaunchKernelGGL((kv_append8_kernel<LG, true>), grid, dim3(256), 0, st, a, q_blocks);
        else hipLaunchKernelGGL((kv_append8_kernel<LG, false>), grid, dim3(256), 0, st, a, q_blocks);
    });
}

bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// ------------------------------------------------------------- reading back

// A workgroup a token, 8 values a lane.
template <bool CODES>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
    const int t = static_cast<int>(a.first + blockIdx.x);
    const int s = seq_of(a.batch, t);
    if (s < 0) return;
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count) return;
    const int pos = q.keys - q.count + (t - q.start);
    const int P = a.batch.prefix_len, D = a.cache.dim, Hk = a.cache.heads;
    int page = -1, row = 0;
    if (pos >= 0) {
        const int32_t* table = pos < P ? a.batch.prefix_table : a.batch.page_table + static_cast<size_t>(s) * a.batch.table_width;
        const int i = pos < P ? pos : pos - P;
        page = table[i >> a.cache.page_shift];
        row = i & ((1 << a.cache.page_shift) - 1);
    }
    const bool there = page >= 0 && page < a.cache.num_pages;
    const uint32_t fill = pos < 0 ? 0u : 0xffffffffu;          // NaN in fp16 and bf16
    const int each = Hk * D / 8;
    for (int i = threadIdx.x; i < 2 * each; i += 256) {
        const bool is_v = i >= each;
        const int at = 8 * (is_v ? i - each : i), head = at / D;
        u32x4 x = {fill, fill, fill, fill};
        if (there) {
            const int r = ((page * Hk + head) << a.cache.page_shift) + row;
            const size_t from = static_cast<size_t>(r) * D + at % D;
            if constexpr (CODES) {
                const uint32_t b = (is_v ? a.cache.v_scale : a.cache.k_scale)[static_cast<unsigned>(r) >> a.cache.block_shift];
                const float scale = __builtin_bit_cast(float, b << 23);
                const u32x2 c = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(is_v ? a.cache.v : a.cache.k) + from);
                const f32x2 v[4] = {__builtin_amdgcn_cvt_pk_f32_fp8(c[0], false), __builtin_amdgcn_cvt_pk_f32_fp8(c[0], true),
                                    __builtin_amdgcn_cvt_pk_f32_fp8(c[1], false), __builtin_amdgcn_cvt_pk_f32_fp8(c[1], true)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Quad two{{v[j][0] * scale, v[j][1] * scale, 0.f, 0.f}};
                    x[j] = narrow(two, a.cache.dtype).a;
                }
            } else {
                x = *reinterpret_cast<const u32x4*>((is_v ? a.cache.v : a.cache.k) + from);
            }
        }
        *reinterpret_cast<u32x4*>((is_v ? a.v : a.k) + static_cast<size_t>(t) * Hk * D + at) = x;
    }
}

}  // namespace

hipError_t launch_kv_append8(const AppendArgs& a, hipStream_t st) {
    const bool vec = wide(a.q) && wide(a.k) && wide(a.v) && wide(a.q_out) && wide(a.q_norm) && wide(a.k_norm) &&
                     a.q_stride % 8 == 0 && a.k_stride % 8 == 0 && a.v_stride % 8 == 0;
    if (a.cache.dim <= 64) return launch<8>(a, vec, st);
    if (a.cache.dim <= 128) return launch<16>(a, vec, st);
    return launch<32>(a, vec, st);
}

hipError_t launch_kv_read(const ReadArgs& args, bool codes, hipStream_t st) {
    ReadArgs a = args;
    return launch_all(a.batch.tokens, [&](unsigned first, unsigned count) {
        a.first = first;
        if (codes) hipLaunchKernelGGL((kv_read_kernel<true>), dim3(count), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((kv_read_kernel<false>), dim3(count), dim3(256), 0, st, a);
    });
}

}  // namespace cl
