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

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {
namespace {

// VEC consecutive elements of an fp16, bf16 or fp32 array as fp32.
template <int VEC>
__device__ __forceinline__ void load_vec(const void* p, size_t i, int dt, float* o) {
    if constexpr (VEC == 8) {
        if (dt == DT_FP32) {
            const f32x4* f = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
            const f32x4 a = f[0], b = f[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = a[j], o[4 + j] = b[j];
        } else {
            const u32x4 u = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t uj = u[j];
                o[2 * j] = act_to_f32(static_cast<uint16_t>(uj & 0xffff), dt);
                o[2 * j + 1] = act_to_f32(static_cast<uint16_t>(uj >> 16), dt);
            }
        }
    } else {
        o[0] = dt == DT_FP32 ? static_cast<const float*>(p)[i] : act_to_f32(static_cast<const uint16_t*>(p)[i], dt);
    }
}

template <int VEC>
__device__ __forceinline__ void store_vec(void* p, size_t i, int dt, const float* v) {
    if constexpr (VEC == 8) {
        if (dt == DT_FP32) {
            f32x4* f = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
            f[0] = f32x4{v[0], v[1], v[2], v[3]};
            f[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            u32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t lo = dt == DT_FP16 ? f32_to_f16_bits(v[2 * j]) : f32_to_bf16_bits(v[2 * j]);
                const uint32_t hi = dt == DT_FP16 ? f32_to_f16_bits(v[2 * j + 1]) : f32_to_bf16_bits(v[2 * j + 1]);
                u[j] = lo | hi << 16;
            }
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) = u;
        }
    } else {
        store_out(p, i, v[0], dt);
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

// x <- N(x) over the row; elements past d stay zero.
template <int VEC, int NI>
__device__ __forceinline__ void normalise(float (&x)[NI][VEC], const bool (&live)[NI], const NormArgs& a,
                                          float (*slots)[16]) {
    if (a.layer) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s += x[i][j];
        const float mean = block_sum(s, slots[0]) / static_cast<float>(a.d);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (live[i]) x[i][j] -= mean;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += x[i][j] * x[i][j];
    const float r = 1.0f / sqrtf(block_sum(s, slots[1]) / static_cast<float>(a.d) + a.eps);
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[i][j] *= r;
}

template <int VEC, int NI>
__global__ void residual_norm_kernel(NormArgs a) {
    __shared__ float slots[4][16];
    const int t = blockIdx.x;
    const size_t row = static_cast<size_t>(t) * a.d;
    float x[NI][VEC];
    int at[NI];
    bool live[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        at[i] = (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * VEC;
        live[i] = at[i] < a.d;
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[i][j] = 0.f;
    }
    if (a.slots) {
#pragma unroll 4
        for (int s = 0; s < a.slots; ++s) {
            const float w = a.slot_weights[static_cast<size_t>(t) * a.slots + s];
            const size_t base = (static_cast<size_t>(t) * a.slots + s) * a.d;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (live[i]) {
                    float y[VEC];
                    load_vec<VEC>(a.y, base + at[i], a.y_dtype, y);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[i][j] += w * y[j];
                }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (live[i]) load_vec<VEC>(a.y, row + at[i], a.y_dtype, x[i]);
    }
    if (a.post_weight) {
        normalise<VEC, NI>(x, live, a, slots);
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (live[i]) {
                float w[VEC];
                load_vec<VEC>(a.post_weight, at[i], a.w_dtype, w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[i][j] *= w[j];
            }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
        if (live[i]) {
            if (a.gate) {
                float g[VEC];
                load_vec<VEC>(a.gate, a.gate_per_token ? row + at[i] : at[i], a.w_dtype, g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[i][j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[i][j] *= a.beta;
            if (a.residual) {
                float r[VEC];
                load_vec<VEC>(a.residual, row + at[i], a.h_dtype, r);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[i][j] = fmaf(a.alpha, r[j], x[i][j]);
            }
            if (a.h) store_vec<VEC>(a.h, row + at[i], a.h_dtype, x[i]);
        }
    normalise<VEC, NI>(x, live, a, slots + 2);
#pragma unroll
    for (int i = 0; i < NI; ++i)
        if (live[i]) {
            float w[VEC];
            load_vec<VEC>(a.weight, at[i], a.w_dtype, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[i][j] *= w[j];
            if (a.bias) {
                load_vec<VEC>(a.bias, at[i], a.w_dtype, w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[i][j] += w[j];
            }
            store_vec<VEC>(a.out, row + at[i], a.out_dtype, x[i]);
        }
}

template <int VEC, int NI>
hipError_t launch(const NormArgs& a, hipStream_t st) {
    const int lanes = (a.d + VEC * NI - 1) / (VEC * NI);
    const int threads = (lanes + 63) / 64 * 64;
    hipLaunchKernelGGL((residual_norm_kernel<VEC, NI>), dim3(a.T), dim3(threads), 0, st, a);
    return hipGetLastError();
}

bool vec_ok(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

hipError_t launch_residual_norm(const NormArgs& a, hipStream_t st) {
    const bool vec = a.d % 8 == 0 && vec_ok(a.y) && vec_ok(a.residual) && vec_ok(a.weight) && vec_ok(a.bias) &&
                     vec_ok(a.post_weight) && vec_ok(a.gate) && vec_ok(a.h) && vec_ok(a.out);
    if (vec) {
        if (a.d <= 8192) return launch<8, 1>(a, st);
        if (a.d <= 16384) return launch<8, 2>(a, st);
        return launch<8, 4>(a, st);
    }
    if (a.d <= 4096) return launch<1, 4>(a, st);
    return launch<1, 32>(a, st);
}

}  // namespace cl
