// Routing of tokens to experts: scores, groups, the k best, their weights and
// the ranks of their compensation factors.
//
//     s_e = e^{l_e - max} / sum   or   1 / (1 + e^{-l_e});   c_e = s_e + bias_e
//
// Without a bias the logits themselves are compared (both scores rise with
// the logit, and equal scores of unequal logits would decide by rounding).
// A wave owns a token and holds its experts in registers, expert e in lane
// e % 64, so a token's logits are read once and nothing is exchanged through
// memory.  Values become unsigned keys of the same order; each of the k steps
// takes the wave's largest key by DPP (no LDS round trip) and finds the lowest
// expert that holds it by one ballot per 64 experts.  Bound by latency: 64 tokens
// of 128 experts, 8 chosen, 4.5 us, of which a launch is 3, and 0.4 us for each
// table of ranks (loads that wait for the choice); 4099 tokens of 256 in groups 9 us.

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {
namespace {

// Keys: larger for larger floats; every number is at least 0x007fffff (-inf).
// A NaN logit stands behind a NaN score: one NaN logit makes every score of a
// softmax NaN, and it is still the last to be chosen.
constexpr uint32_t kTaken = 0, kClosed = 1, kNaN = 2, kNaNScore = 3;

__device__ __forceinline__ uint32_t order_key(float v, uint32_t nan = kNaN) {
    if (v != v) return nan;
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);   // -0 compares equal to 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false);
    return v > o ? v : o;
}

// Largest value of the wave, in every lane (a scalar).
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = dpp_max<0x111>(v);      // row_shr 1, 2, 4, 8: lane 15 of each row of 16 has the row's
    v = dpp_max<0x112>(v);
    v = dpp_max<0x114>(v);
    v = dpp_max<0x118>(v);
    v = dpp_max<0x142>(v);      // row_bcast 15, 31: lane 63 has the wave's
    v = dpp_max<0x143>(v);
    return __builtin_amdgcn_readlane(static_cast<int>(v), 63);
}

template <int EPL>
__global__ __launch_bounds__(256) void moe_route_kernel(RouteArgs a) {
    __shared__ float group_choice[4][EPL > 1 ? 64 * EPL : 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned t = 4 * (a.first + blockIdx.x) + wave;
    if (t >= static_cast<unsigned>(a.T)) return;

    float p[EPL];
    uint32_t key[EPL];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        const int e = 64 * i + lane;
        p[i] = -INFINITY;
        if (e < a.E) {
            const size_t at = static_cast<size_t>(t) * a.E + e;
            p[i] = a.dtype == DT_FP32 ? static_cast<const float*>(a.logits)[at]
                                      : act_to_f32(static_cast<const uint16_t*>(a.logits)[at], a.dtype);
        }
        key[i] = e < a.E ? order_key(p[i]) : kTaken;
        m = fmaxf(m, p[i]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) p[i] = 1.0f / (1.0f + expf(-p[i]));
    } else {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            // a row of -inf alone has no probability to share: scores of 0
            p[i] = m == -INFINITY && p[i] == m ? 0.f : expf(p[i] - m);
            if (64 * i + lane >= a.E) p[i] = 0.f;
            s += p[i];
        }
        s = wave_sum(s);
        if (s != 0.f) {
#pragma unroll
            for (int i = 0; i < EPL; ++i) p[i] = p[i] / s;
        }
    }
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int e = 64 * i + lane;
            if (e < a.E && key[i] != kNaN) key[i] = order_key(p[i] + a.bias[e], kNaNScore);
        }
    }

    if (a.groups > 1) {
        // c of every expert to the wave's own LDS row (the key back as a float;
        // a sum of two without a bias takes the scores), then the groups'
        // best one or two are found
        const bool scores = a.group_best == 2 && !a.bias;
        float* c = group_choice[wave];
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const uint32_t u = key[i];
            const float v = u <= kNaNScore ? -INFINITY
                            : scores  ? p[i]
                                      : __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u);
            c[64 * i + lane] = v;
        }
        __builtin_amdgcn_wave_barrier();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // `per` neighbouring lanes share a group and each scans every per-th of
        // its values; the pairs of best ones meet by shuffles
        const int size = a.E / a.groups;
        int per = 64;
        while (per * a.groups > 64) per >>= 1;
        const int mine = lane / per;
        float b1 = -INFINITY, b2 = -INFINITY;
        if (mine < a.groups) {
#pragma unroll 4
            for (int j = lane % per; j < size; j += per) {
                const float v = c[mine * size + j];
                b2 = fmaxf(b2, fminf(b1, v));
                b1 = fmaxf(b1, v);
            }
        }
        for (int off = 1; off < per; off <<= 1) {
            const float o1 = __shfl_xor(b1, off, 64), o2 = __shfl_xor(b2, off, 64);
            b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
            b1 = fmaxf(b1, o1);
        }
        // lane g carries on for group g
        b1 = __shfl(b1, min(lane * per, 63), 64);
        b2 = __shfl(b2, min(lane * per, 63), 64);
        uint32_t gk = lane < a.groups ? order_key(a.group_best == 2 && size > 1 ? b1 + b2 : b1) : kTaken;
        uint64_t open = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            const uint32_t best = wave_max_u32(gk);
            const int g = __ffsll(static_cast<unsigned long long>(__ballot(gk == best && lane < a.groups && !((open >> lane) & 1)))) - 1;
            open |= 1ull << g;
            if (lane == g) gk = kTaken;
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int e = 64 * i + lane;
            if (e < a.E && !((open >> (e / size)) & 1)) key[i] = kClosed;
        }
    }

    int id = 0;
    float w = 0.f;
    for (int j = 0; j < a.k; ++j) {
        uint32_t mine = key[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) mine = mine > key[i] ? mine : key[i];
        const uint32_t best = wave_max_u32(mine);
        bool found = false;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const uint64_t has = __ballot(key[i] == best);
            if (!found && has) {
                found = true;
                const int l = __ffsll(static_cast<unsigned long long>(has)) - 1;
                const float pw = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p[i]), l));
                if (lane == j) id = 64 * i + l, w = pw;
                if (lane == l) key[i] = kTaken;
            }
        }
    }
    if (a.renormalize) {
        const float s = wave_sum(lane < a.k ? w : 0.f);
        if (s != 0.f) w = w / s;
    }
    w *= a.scale;
    if (lane >= a.k) return;
    const size_t at = static_cast<size_t>(t) * a.k + lane;
    a.ids[at] = id;
    a.weights[at] = w;
    // the level nearest to k w r, ties to the lower; fp64, as the host's rule
    for (int n = 0; n < a.tables; ++n) {
        const double x = static_cast<double>(a.k) * static_cast<double>(w) * static_cast<double>(a.expert_ranks[n][id]);
        int best = a.levels[0];
        for (int l = 1; l < a.nlevels; ++l)
            if (fabs(x - a.levels[l]) < fabs(x - best)) best = a.levels[l];
        a.slot_ranks[n][at] = best;
    }
}

}  // namespace

hipError_t launch_moe_route(RouteArgs a, hipStream_t st) {
    return launch_all((static_cast<long long>(a.T) + 3) / 4, [&](unsigned first, unsigned count) {
        a.first = first;
        const dim3 grid(count), block(256);
        if (a.E <= 64) hipLaunchKernelGGL((moe_route_kernel<1>), grid, block, 0, st, a);
        else if (a.E <= 128) hipLaunchKernelGGL((moe_route_kernel<2>), grid, block, 0, st, a);
        else if (a.E <= 256) hipLaunchKernelGGL((moe_route_kernel<4>), grid, block, 0, st, a);
        else if (a.E <= 512) hipLaunchKernelGGL((moe_route_kernel<8>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((moe_route_kernel<16>), grid, block, 0, st, a);
    });
}

}  // namespace cl
