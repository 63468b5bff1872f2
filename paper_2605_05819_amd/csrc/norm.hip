// A block's output into the residual stream, and the next block's input:
//
//     u = sum_j w_j y_j   (a MoE token's slots)  or  y
//     u <- N(u) post_weight                      (norm after the block)
//     h = alpha residual + beta gate u
//     out = N(h) weight + bias                   (norm before the next block)
//
// N(x) = x / sqrt(mean x^2 + eps), or the same of x - mean x.  One pass over
// memory: a workgroup holds its token's row in registers as fp32 from the load
// to the last store, so every operand is read once and both results are
// written once; the statistics are fp32 sums (the centred norm takes the mean
// first, then the squares of the differences, so no digits cancel), and out is
// formed from the unrounded h.
//
// Bound by memory: 2048 rows of 4096 with post-norm and per-token gate, 84 MB in
// 17.5 us, 4.8 TB/s; 64 tokens of 8 slots by latency, 6 us.  (Asking for
// residual, gate and weights ahead of the sums costs the registers of a wave:
// 24 us.)

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {
namespace {

// Eight 16-bit values, or four floats, at any alignment of their elements (the
// target reads and writes global memory unaligned).
struct __attribute__((packed, aligned(2))) Bytes16 {
    u32x4 v;
};

// Elements i .. i + 7 of an fp16, bf16 or fp32 array as fp32; with TAIL only
// the first n are there, the rest are zero.
template <bool TAIL>
__device__ __forceinline__ void load8(const void* p, size_t i, int dt, int n, float (&o)[8]) {
    if (!TAIL || n == 8) {
        if (dt == DT_FP32) {
            const float* f = static_cast<const float*>(p) + i;
            const u32x4 a = reinterpret_cast<const Bytes16*>(f)->v, b = reinterpret_cast<const Bytes16*>(f + 4)->v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t x = a[j], y = b[j];
                o[j] = __builtin_bit_cast(float, x);
                o[4 + j] = __builtin_bit_cast(float, y);
            }
        } else {
            const u32x4 u = reinterpret_cast<const Bytes16*>(static_cast<const uint16_t*>(p) + i)->v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t uj = u[j];
                o[2 * j] = act_to_f32(static_cast<uint16_t>(uj & 0xffff), dt);
                o[2 * j + 1] = act_to_f32(static_cast<uint16_t>(uj >> 16), dt);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            o[j] = j >= n            ? 0.f
                   : dt == DT_FP32 ? static_cast<const float*>(p)[i + j]
                                   : act_to_f32(static_cast<const uint16_t*>(p)[i + j], dt);
    }
}

// STREAM: a prompt's results (2^20 values on) are stored past the L2 caches
// (2048 x 4096 with post-norm and gate 18.8 -> 17.2 us when it was changed).  A
// linear of 4096 behind the call is no slower for it: 1500 rows, both, 89.1 us
// against 89.7 with ordinary stores, 3000 146.6 / 145.8, 8593 384 / 384.
template <bool STREAM>
__device__ __forceinline__ void put(void* p, u32x4 v) {
    Bytes16* const to = static_cast<Bytes16*>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(v, &to->v);
    else to->v = v;
}

template <bool TAIL, bool STREAM>
__device__ __forceinline__ void store8(void* p, size_t i, int dt, int n, const float (&v)[8]) {
    if (!TAIL || n == 8) {
        if (dt == DT_FP32) {
            float* f = static_cast<float*>(p) + i;
            u32x4 a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = __builtin_bit_cast(uint32_t, v[j]);
                b[j] = __builtin_bit_cast(uint32_t, v[4 + j]);
            }
            put<STREAM>(f, a);
            put<STREAM>(f + 4, b);
        } else {
            u32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t lo = dt == DT_FP16 ? f32_to_f16_bits(v[2 * j]) : f32_to_bf16_bits(v[2 * j]);
                const uint32_t hi = dt == DT_FP16 ? f32_to_f16_bits(v[2 * j + 1]) : f32_to_bf16_bits(v[2 * j + 1]);
                u[j] = lo | hi << 16;
            }
            put<STREAM>(static_cast<uint16_t*>(p) + i, u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) store_out(p, i + j, v[j], dt);
    }
}

// Sum over the workgroup, in wave order; `slot` is a fresh LDS row per call.
__device__ __forceinline__ float block_sum(float v, float* slot) {
    v = wave_sum(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += slot[w];
    return s;
}

// x <- N(x) over the row; a lane's pieces hold n[i] elements, the rest stay zero.
template <int NI, bool TAIL>
__device__ __forceinline__ void normalise(float (&x)[NI][8], const int (&n)[NI], const NormArgs& a, float (*slots)[16]) {
    if (a.layer) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[i][j];
        const float mean = block_sum(s, slots[0]) / static_cast<float>(a.d);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = (TAIL ? j < n[i] : n[i] > 0) ? x[i][j] - mean : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += x[i][j] * x[i][j];
    const float r = 1.0f / sqrtf(block_sum(s, slots[1]) / static_cast<float>(a.d) + a.eps);
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] *= r;
}

template <int NI, bool TAIL, bool STREAM>
__global__ void residual_norm_kernel(NormArgs a) {
    __shared__ float slots[4][16];
    const int t = blockIdx.x;
    const size_t row = static_cast<size_t>(t) * a.d;
    float x[NI][8], w[8];
    int at[NI], n[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        at[i] = (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
        n[i] = min(max(a.d - at[i], 0), 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    }
    if (a.slots) {
#pragma unroll 4
        for (int s = 0; s < a.slots; ++s) {
            const float ws = a.slot_weights[static_cast<size_t>(t) * a.slots + s];
            const size_t base = (static_cast<size_t>(t) * a.slots + s) * a.d;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (n[i]) {
                    float y[8];
                    load8<TAIL>(a.y, base + at[i], a.y_dtype, n[i], y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[i][j] += ws * y[j];
                }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (n[i]) load8<TAIL>(a.y, row + at[i], a.y_dtype, n[i], x[i]);
    }
    if (a.post_weight) {
        normalise<NI, TAIL>(x, n, a, slots);
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (n[i]) {
                load8<TAIL>(a.post_weight, at[i], a.w_dtype, n[i], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] *= w[j];
            }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
        if (n[i]) {
            if (a.gate) {
                load8<TAIL>(a.gate, a.gate_per_token ? row + at[i] : at[i], a.w_dtype, n[i], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] *= w[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] *= a.beta;
            if (a.residual) {
                load8<TAIL>(a.residual, row + at[i], a.h_dtype, n[i], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = fmaf(a.alpha, w[j], x[i][j]);
            }
            if (a.h) store8<TAIL, STREAM>(a.h, row + at[i], a.h_dtype, n[i], x[i]);
        }
    normalise<NI, TAIL>(x, n, a, slots + 2);
#pragma unroll
    for (int i = 0; i < NI; ++i)
        if (n[i]) {
            load8<TAIL>(a.weight, at[i], a.w_dtype, n[i], w);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] *= w[j];
            if (a.bias) {
                load8<TAIL>(a.bias, at[i], a.w_dtype, n[i], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] += w[j];
            }
            store8<TAIL, STREAM>(a.out, row + at[i], a.out_dtype, n[i], x[i]);
        }
}

template <int NI, bool TAIL>
hipError_t launch(NormArgs a, hipStream_t st) {
    const int lanes = (a.d + 8 * NI - 1) / (8 * NI);
    const int threads = (lanes + 63) / 64 * 64;
    const bool stream = static_cast<long long>(a.T) * a.d >= 1 << 20;
    // a later launch takes its rows' arrays
    const auto at = [](const void* p, size_t n, int dt) {
        return p ? const_cast<char*>(static_cast<const char*>(p)) + n * (dt == DT_FP32 ? 4 : 2) : nullptr;
    };
    const NormArgs all = a;
    return launch_all(a.T, [&](unsigned first, unsigned count) {
        const size_t n = static_cast<size_t>(first) * a.d;
        a.y = at(all.y, a.slots ? n * a.slots : n, a.y_dtype);
        if (a.slots) a.slot_weights = all.slot_weights + static_cast<size_t>(first) * a.slots;
        if (a.gate_per_token) a.gate = at(all.gate, n, a.w_dtype);
        a.residual = at(all.residual, n, a.h_dtype);
        a.h = at(all.h, n, a.h_dtype);
        a.out = at(all.out, n, a.out_dtype);
        if (stream) hipLaunchKernelGGL((residual_norm_kernel<NI, TAIL, true>), dim3(count), dim3(threads), 0, st, a);
        else hipLaunchKernelGGL((residual_norm_kernel<NI, TAIL, false>), dim3(count), dim3(threads), 0, st, a);
    });
}

template <bool TAIL>
hipError_t choose(const NormArgs& a, hipStream_t st) {
    if (a.d <= 4096) return launch<1, TAIL>(a, st);
    if (a.d <= 8192) return launch<2, TAIL>(a, st);
    return launch<4, TAIL>(a, st);
}

}  // namespace

// Pieces of 8 a lane: one up to 512 threads, two up to 8192 values (3000 rows of
// 5000: 35 us, 45 with 640 threads of one piece; 2048 rows of 4096 18.8 with one,
// 20.0 with two).  A width that is no multiple of 8 ends in a shorter piece
// (1000 rows of 4001: 9.2 us; 25 an element at a time).
hipError_t launch_residual_norm(const NormArgs& a, hipStream_t st) {
    return a.d % 8 ? choose<true>(a, st) : choose<false>(a, st);
}

}  // namespace cl
