// A beam search's step: the best continuations of each group's beams.
//
//     s[b][v] = score_b + l[b][v] - ln sum_v e^{l[b][v]},   rank = s / length^alpha
//
// Within a beam the ranks fall with the logits, so a beam's candidates are its
// largest logits (ties to the lower token), and only their order across beams
// needs the sum.  Two launches:
//
//  * beam_scan: a workgroup takes a chunk of a row into registers, once: its sum of
//    exponentials and its k best logits.  Where each of the four waves has k / 4
//    lanes whose maxima reach a bound, k values do; what reaches the least of the
//    waves' k / 4-th largest lane maxima (two or three times k values as a rule) goes to
//    a list in LDS, where each counts how many stand ahead of it.  Where ties with that
//    bound fill the list (masked vocabularies: 27 us for 128 rows of 128000, 21 unmasked)
//    it takes what is above the bound, and the lowest tokens at it.
//  * beam_pick: a workgroup a group: sums joined per beam in fp64, a beam's k best
//    from its chunks' (a lane walks a chunk's list), then the ranks in fp64, each
//    candidate counting those ahead of it.
//
// The sums (and a length's power, off by some 2^-51) are the only rounding that can change an order.  e^l is 2^(l log2 e)
// with what the product's rounding leaves out, and what log2 e lacks in fp32, to first
// order; nothing is taken from l ahead of it where no exponential can overflow or
// vanish (a chunk's largest logit in -32..64), so that nothing else is rounded.  The instruction
// is off by 2^-23.5 at most (measured over its range; -2^-28 on the mean), eight terms are
// added in fp32 as a tree, the rest in fp64: a row's logarithm is off by 2^-21.8 at most, where all
// terms round alike, and by 2^-25 (root mean square; sharp rows of 2000) to 2^-29 (flat ones of 128000)
// where they do not.
// Bound by the read of the logits and by the issue of about fourteen instructions a
// value (the exponential counts four): 128 rows of 128000 in bf16 13.4 us (12.2 with a
// plain 2^(l log2 e - top log2 e), off by 2^-21), in fp32 16.8.

#include <math.h>

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {
namespace {

typedef unsigned long long u64;

constexpr double kLog2e = 1.4426950408889634, kLn2 = 0.69314718055994531;
constexpr float kLog2eHi = static_cast<float>(kLog2e), kLog2eLo = static_cast<float>(kLog2e - kLog2eHi);
constexpr int kList = 1024;                  // entries of a workgroup's list
constexpr int kMaxSplits = 64;               // a lane each in beam_pick

// Larger for larger floats (no NaN among them); every number is above 0.
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.0f);   // -0 compares equal to 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_key(uint32_t k) {
    return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// Value and token, the larger for the larger value, then for the lower token.
__device__ __forceinline__ u64 candidate(float v, int token) {
    return static_cast<u64>(order_key(v)) << 32 | static_cast<uint32_t>(~token);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false);
    return v > o ? v : o;
}
// Largest value of the wave, in every lane (a scalar).
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = dpp_max<0x111>(v);      // row_shr 1, 2, 4, 8, then row_bcast 15, 31
    v = dpp_max<0x112>(v);
    v = dpp_max<0x114>(v);
    v = dpp_max<0x118>(v);
    v = dpp_max<0x142>(v);
    v = dpp_max<0x143>(v);
    return __builtin_amdgcn_readlane(static_cast<int>(v), 63);
}
__device__ __forceinline__ u64 wave_max_u64(u64 v) {
    const uint32_t hi = wave_max_u32(static_cast<uint32_t>(v >> 32));
    const uint32_t lo = wave_max_u32(static_cast<uint32_t>(v >> 32) == hi ? static_cast<uint32_t>(v) : 0u);
    return static_cast<u64>(hi) << 32 | lo;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// 16 bytes at any address that is aligned to its elements.
struct Wide {
    uint32_t w[4];
} __attribute__((packed, aligned(2)));

// ---------------------------------------------------------------- the logits

// A lane holds EPT values: VEC neighbours (16 bytes) a load, the wave's loads side
// by side, so token(j) rises with j and with the lane inside a load.
template <int DT, int EPT>
__global__ __launch_bounds__(256, 8) void beam_scan_kernel(BeamArgs a) {
    constexpr int VEC = DT == DT_FP32 ? 4 : 8, LOADS = EPT / VEC;
    __shared__ u64 list[kList];
    __shared__ int filled;
    __shared__ float tops[4];
    __shared__ uint32_t bounds[4];
    __shared__ double sums[256];
    __shared__ u64 best[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    if (a.finished && a.finished[row]) return;
    const int base = split * a.chunk + wave * 64 * EPT;
    const size_t size = DT == DT_FP32 ? 4 : 2;
    const char* const from = static_cast<const char*>(a.logits) + static_cast<size_t>(row) * a.stride * size;
    const auto token = [&](int j) { return base + (j / VEC) * 64 * VEC + lane * VEC + j % VEC; };

    const bool full = split * a.chunk + a.chunk <= a.vocab;
    float x[EPT], group[LOADS];
    Wide raw[LOADS];
    const auto value = [&](const Wide& w, int j) {
        if constexpr (DT == DT_FP32) return __builtin_bit_cast(float, w.w[j]);
        else return act_to_f32(static_cast<uint16_t>(j & 1 ? w.w[j / 2] >> 16 : w.w[j / 2]), DT);
    };
    if (full) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) raw[i] = *reinterpret_cast<const Wide*>(from + static_cast<size_t>(token(i * VEC)) * size);
    } else {
        // whole pieces, then the row's last values one by one into theirs
        const uint32_t none = DT == DT_FP32 ? 0xff800000u : DT == DT_BF16 ? 0xff80ff80u : 0xfc00fc00u;      // -inf
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            raw[i] = Wide{{none, none, none, none}};
            if (token(i * VEC) + VEC <= a.vocab)
                raw[i] = *reinterpret_cast<const Wide*>(from + static_cast<size_t>(token(i * VEC)) * size);
        }
#pragma unroll 1
        for (int i = 0; i < LOADS; ++i) {
            const int t = token(i * VEC);
            if (t >= a.vocab || t + VEC <= a.vocab) continue;
            Wide w = {{none, none, none, none}};
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (t + j < a.vocab) {
                    if constexpr (DT == DT_FP32) {
                        w.w[j] = reinterpret_cast<const uint32_t*>(from)[t + j];
                    } else {
                        const uint32_t h = reinterpret_cast<const uint16_t*>(from)[t + j];
                        w.w[j / 2] = j & 1 ? (w.w[j / 2] & 0xffffu) | h << 16 : (w.w[j / 2] & 0xffff0000u) | h;
                    }
                }
#pragma unroll
            for (int n = 0; n < LOADS; ++n)
                if (n == i) raw[n] = w;
        }
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[i * VEC + j] = value(raw[i], j);
    // (a NaN makes the sum NaN, and the row has no list then; the maxima only have
    // to take it without more instructions)
    float mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        group[i] = x[i * VEC];
#pragma unroll
        for (int j = 1; j < VEC; ++j) group[i] = __builtin_elementwise_maximum(group[i], x[i * VEC + j]);
        mine = __builtin_elementwise_maximum(mine, group[i]);
    }
    // lane maxima one after another: k / 4 of each wave, and the least of the
    // waves' last ones; in a row's last chunk, where waves may be empty, k of each,
    // and the largest
    const int each = full ? (a.picks + 3) / 4 : a.picks;
    uint32_t key = token(0) < a.vocab ? order_key(mine != mine ? -INFINITY : mine) : 0u, kth = 0;
    for (int j = 0; j < each; ++j) {
        kth = wave_max_u32(key);
        if (j == 0 && lane == 0) tops[wave] = kth ? from_key(kth) : -INFINITY;
        const uint64_t has = __ballot(key == kth);
        if (lane == __ffsll(static_cast<unsigned long long>(has)) - 1) key = 0;
    }
    if (lane == 0) bounds[wave] = kth;
    if (tid == 0) filled = 0;
    __syncthreads();
    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    uint32_t bound = bounds[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) bound = full ? min(bound, bounds[w]) : max(bound, bounds[w]);
    const float least = bound ? from_key(bound) : -INFINITY;

    // the sum of e^(x - reference), as 2^p with what p lacks beside it; far below the
    // reference (-inf too) is 0, and a NaN or an infinity makes the row's sum NaN
    const bool near = top >= -32.0f && top <= 64.0f;      // reference 0
    const double zero = near ? 0.0 : static_cast<double>(top);
    double s = 0.0;
    float more = 0.f;
    const auto add = [&](int i, auto form) {
        float e[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float p, rest;
            form(x[i * VEC + j], p, rest);
            e[j] = __builtin_amdgcn_exp2f(p);
            more = fmaf(e[j], rest, more);
        }
#pragma unroll
        for (int w = VEC / 2; w > 0; w /= 2)
#pragma unroll
            for (int j = 0; j < w; ++j) e[j] += e[j + w];
        s += static_cast<double>(e[0]);
    };
    if (near) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            add(i, [](float l, float& p, float& rest) {
                l = fmaxf(l, -200.f);
                p = l * kLog2eHi;
                rest = fmaf(l, kLog2eLo, fmaf(l, kLog2eHi, -p));
            });
    } else {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            add(i, [zero](float l, float& p, float& rest) {
                const double d = fmax(static_cast<double>(l) - zero, -200.0) * kLog2e;
                p = static_cast<float>(d);
                rest = static_cast<float>(d - static_cast<double>(p));
            });
    }
    s = mine != mine || top == INFINITY ? static_cast<double>(NAN) : s + static_cast<double>(more) * kLn2;
    sums[tid] = s;

    // those that `fit` to the list, as far as it goes
    const auto collect = [&](auto fit) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (__ballot(fit(group[i]))) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (fit(x[i * VEC + j]) && token(i * VEC + j) < a.vocab) {
                        const int at = atomicAdd(&filled, 1);
                        if (at < kList) list[at] = candidate(x[i * VEC + j], token(i * VEC + j));
                    }
            }
    };
    collect([least](float v) { return v >= least; });
    __syncthreads();
    const size_t slot = static_cast<size_t>(row) * a.splits + split;
    u64* const out = a.best + slot * a.picks;
    if (wave == 3) {
        const double total = wave_sum(sums[lane] + sums[lane + 64] + sums[lane + 128] + sums[lane + 192]);
        if (lane == 0) {
            a.sum[slot] = total;
            a.most[slot] = zero;
        }
    }
    int n = filled;
    if (n > kList) {
        // ties with the least (masks, as a rule): those above it, then its lowest tokens one after another
        uint32_t equal = 0;                            // of the lane's values
#pragma unroll
        for (int j = 0; j < EPT; ++j) equal |= x[j] == least && token(j) < a.vocab ? 1u << j : 0u;
        __syncthreads();
        if (tid == 0) filled = 0;
        __syncthreads();
        collect([least](float v) { return v > least; });
        __syncthreads();
        n = filled;
        while (n < a.picks) {
            const uint32_t key = equal ? ~static_cast<uint32_t>(token(__ffs(static_cast<int>(equal)) - 1)) : 0u;
            const uint32_t most = wave_max_u32(key);
            if (lane == 0) bounds[wave] = most;
            __syncthreads();
            const uint32_t c = max(max(bounds[0], bounds[1]), max(bounds[2], bounds[3]));
            if (c == 0) break;                         // all values of a row's end
            if (key == c) equal &= equal - 1;
            if (tid == 0) list[n] = static_cast<u64>(order_key(least)) << 32 | c;
            ++n;
            __syncthreads();
        }
    }
    if (n <= kList) {
        for (int i = tid; i < n; i += 256) {
            const u64 c = list[i];
            int ahead = 0;
            for (int j = 0; j < n; ++j) ahead += list[j] > c;
            if (ahead < a.picks) out[ahead] = c;
        }
        for (int i = n + tid; i < a.picks; i += 256) out[i] = 0;      // fewer values than picks
        return;
    }
    // more than the list holds above the least lane's maximum: each next best below the last
    // one, from memory again (values held for this would cost every chunk its registers)
    u64 last = ~0ull;
    for (int k = 0; k < a.picks; ++k) {
        u64 c = 0;
#pragma unroll 1
        for (int i = 0; i < LOADS; ++i) {
            const int t = token(i * VEC);
            const auto take = [&](float v, int at) {
                const u64 o = candidate(v, at);
                if (o < last && o > c) c = o;
            };
            if (t + VEC <= a.vocab) {
                const Wide w = *reinterpret_cast<const Wide*>(from + static_cast<size_t>(t) * size);
#pragma unroll
                for (int j = 0; j < VEC; ++j) take(value(w, j), t + j);
            } else {
                for (int j = t; j < a.vocab; ++j) {
                    if constexpr (DT == DT_FP32) take(reinterpret_cast<const float*>(from)[j], j);
                    else take(act_to_f32(reinterpret_cast<const uint16_t*>(from)[j], DT), j);
                }
            }
        }
        c = wave_max_u64(c);
        if (lane == 0) best[wave] = c;
        __syncthreads();
        last = best[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) last = last > best[w] ? last : best[w];
        if (tid == 0) out[k] = last;
        __syncthreads();
    }
}

// ------------------------------------------------------------------ the picks

// Larger for larger ranks; NaN behind -inf.
__device__ __forceinline__ u64 rank_key(double v) {
    if (v != v) return 1;
    const u64 u = __builtin_bit_cast(u64, v + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

constexpr int kPick = 1024;

// LDS: the candidates of a group, beams x picks of them, descending within a beam:
// rank, score, token; then a list of splits x picks for each wave.
__global__ __launch_bounds__(kPick) void beam_pick_kernel(BeamArgs a, int waves) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int n = a.beams * a.picks;
    u64* const rank = reinterpret_cast<u64*>(lds);
    u64* const lists = rank + n;
    float* const score = reinterpret_cast<float*>(lists + static_cast<size_t>(waves) * a.splits * a.picks);
    int* const token = reinterpret_cast<int*>(score + n);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = blockIdx.x;

    if (wave < waves)
        for (int b = wave; b < a.beams; b += waves) {
            const int row = g * a.beams + b;
            const bool done = a.finished && a.finished[row];
            const int len = (a.lengths ? a.lengths[row] : 0) + (done ? 0 : 1);
            // the lists' loads go ahead of the sums' chain
            u64* const mine = lists + static_cast<size_t>(wave) * a.splits * a.picks;
            const u64* const from = a.best + static_cast<size_t>(row) * a.splits * a.picks;
            if (!done)
                for (int i = lane; i < a.splits * a.picks; i += 64) mine[i] = from[i];
            const double by = a.alpha != 0.0 && len > 1 ? exp(a.alpha * log(static_cast<double>(len))) : 1.0;
            const double before = static_cast<double>(a.scores[row]);
            // all candidates of one score: a finished beam's -inf, a beam of -inf, NaN
            double same = -INFINITY, top = 0.0, lse = 0.0;      // lse: beyond top
            bool plain = done;
            if (!done) {
                const size_t at = static_cast<size_t>(row) * a.splits + lane;
                const double m = lane < a.splits ? a.most[at] : -INFINITY;
                const double s = lane < a.splits ? a.sum[at] : 0.0;
                top = m;
#pragma unroll
                for (int off = 32; off > 0; off >>= 1) top = fmax(top, __shfl_xor(top, off, 64));
                const double sum = wave_sum(s == 0.0 ? 0.0 : s * exp(m - top));
                lse = log(sum);
                if (sum == 0.0) plain = true;                          // no logit above -inf
                if (!(fabs(sum) <= 1.7976931348623157e308) || !(before <= 3.4028234663852886e38)) plain = true, same = NAN;
                else if (before == -INFINITY) plain = true;
            }
            if (plain) {
                // the lowest tokens, a finished beam's own ahead of them
                for (int j = lane; j < a.picks; j += 64) {
                    int v = j;
                    double s = same;
                    if (done && a.eos >= 0) {
                        v = j == 0 ? a.eos : j - 1 < a.eos ? j - 1 : j;
                        if (j == 0) s = before <= 3.4028234663852886e38f ? before : NAN;
                    }
                    rank[b * a.picks + j] = v < a.vocab ? rank_key(s / by) : 0;
                    score[b * a.picks + j] = static_cast<float>(s);
                    token[b * a.picks + j] = v;
                }
                continue;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            int next = 0;
            u64 head = lane < a.splits ? mine[lane * a.picks] : 0;
            for (int j = 0; j < a.picks; ++j) {
                const u64 c = wave_max_u64(head);
                if (head == c && c != 0) {
                    ++next;
                    head = next < a.picks ? mine[lane * a.picks + next] : 0;
                    const double s = before + ((static_cast<double>(from_key(static_cast<uint32_t>(c >> 32))) - top) - lse);
                    rank[b * a.picks + j] = rank_key(s / by);
                    score[b * a.picks + j] = static_cast<float>(s);
                    token[b * a.picks + j] = static_cast<int>(~static_cast<uint32_t>(c));
                }
                if (c == 0 && lane == 0) rank[b * a.picks + j] = 0;     // fewer tokens than picks
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    __syncthreads();
    // the place of every candidate: those of a larger rank, and of an equal one that stand before it
    int per = 1;
    while (per < 64 && 2 * per * n <= kPick) per *= 2;
    const int step = kPick / per;
    for (int first = 0; first < n; first += step) {
        const int i = first + tid / per;
        const u64 r = i < n ? rank[i] : 0;
        int ahead = 0;
        if (i < n)
            for (int j = tid % per; j < n; j += per) ahead += rank[j] > r || (rank[j] == r && j < i);
        for (int off = 1; off < per; off <<= 1) ahead += __shfl_xor(ahead, off, 64);
        if (i >= n || tid % per || ahead >= a.picks || r == 0) continue;
        const int row = g * a.beams + i / a.picks;
        const bool done = a.finished && a.finished[row];
        const size_t at = static_cast<size_t>(g) * a.picks + ahead;
        a.out_scores[at] = score[i];
        a.tokens[at] = token[i];
        a.parents[at] = row;
        if (a.out_lengths) a.out_lengths[at] = a.lengths[row] + (done ? 0 : 1);
        if (a.out_finished) a.out_finished[at] = done || token[i] == a.eos;
    }
}

size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

// A chunk of 256 x EPT values: 2048 where rows are few (their scan is a chain of
// latencies), up to 8192 where they fill the chip (fewer lists to join).
void cut(BeamArgs& a) {
    const long long rows = static_cast<long long>(a.groups) * a.beams;
    a.chunk = 2048;
    while (a.chunk < 8192 && (rows * ((a.vocab + a.chunk - 1) / a.chunk) > 1024 || (a.vocab + a.chunk - 1) / a.chunk > kMaxSplits))
        a.chunk *= 2;
    a.splits = (a.vocab + a.chunk - 1) / a.chunk;
}

size_t pick_lds(const BeamArgs& a, int waves) {
    return static_cast<size_t>(a.beams) * a.picks * 16 + static_cast<size_t>(waves) * a.splits * a.picks * 8;
}

template <int DT>
void scan(const BeamArgs& a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.groups) * a.beams * a.splits);
    if (a.chunk == 2048) hipLaunchKernelGGL((beam_scan_kernel<DT, 8>), grid, dim3(256), 0, st, a);
    else if (a.chunk == 4096) hipLaunchKernelGGL((beam_scan_kernel<DT, 16>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((beam_scan_kernel<DT, 32>), grid, dim3(256), 0, st, a);
}

}  // namespace

// Workgroups of the scan stay below 2^32 work items, chunks of a row within a wave's lanes.
bool beam_fits(const BeamArgs& args) {
    BeamArgs a = args;
    cut(a);
    return a.splits <= kMaxSplits && static_cast<long long>(a.groups) * a.beams * a.splits < (1 << 24);
}

size_t beam_workspace_bytes(BeamArgs a) {
    cut(a);
    const size_t slots = static_cast<size_t>(a.groups) * a.beams * a.splits;
    return up256(slots * a.picks * 8) + 2 * up256(slots * 8);
}

hipError_t launch_beam_select(BeamArgs a, void* ws, hipStream_t st) {
    cut(a);
    const size_t slots = static_cast<size_t>(a.groups) * a.beams * a.splits;
    char* at = static_cast<char*>(ws);
    a.best = reinterpret_cast<u64*>(at);
    at += up256(slots * a.picks * 8);
    a.sum = reinterpret_cast<double*>(at);
    a.most = reinterpret_cast<double*>(at + up256(slots * 8));
    if (a.dtype == DT_FP32) scan<DT_FP32>(a, st);
    else if (a.dtype == DT_BF16) scan<DT_BF16>(a, st);
    else scan<DT_FP16>(a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int waves = a.beams < kPick / 64 ? a.beams : kPick / 64;
    while (waves > 1 && pick_lds(a, waves) > 131072) waves /= 2;
    const size_t bytes = pick_lds(a, waves);
    if (bytes > 65536) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&beam_pick_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(bytes));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(beam_pick_kernel, dim3(a.groups), dim3(kPick), bytes, st, a, waves);
    return hipGetLastError();
}

}  // namespace cl
