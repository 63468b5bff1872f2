// Attention over the paged cache.
//
// Token i of a sequence with n keys and a new tokens stands at p = n - a + i
// and sees key j if j < n, j <= p (causal) and j > p - window (windowed):
//
//     o = sum_j e^{s_j - m} v_j / sum_j e^{s_j - m},  s_j = scale q . k_j,  m = max_j s_j
//
// One pass over the keys with a running maximum and sum.  The rows of a unit
// are the queries that share a key head: token i and head h of the group are
// row i g + h (g = q_heads / kv_heads), 16 rows to an MFMA block.  Both products
// are taken transposed on v_mfma_f32_16x16x32:
//
//     S^T = K Q^T    a lane holds 4 keys of one row (column) per block
//     O^T = V^T P^T  the same lane's probabilities are its operand as they are
//
// Between them no value changes lanes: 16x16x32 sums over 8 keys of each lane
// group g, and which keys these are is free as long as both operands agree, so
// group g takes keys 4g..4g+3 of two neighbouring 16-key blocks, what S^T left
// there.  V^T comes from row-major V in LDS by the transposing read (16 lanes
// turn 4 keys x 16 dims).  Row sums stay per lane until the end; only the
// maximum crosses lanes (two swaps a block).
//
// The keys are two segments, the shared prefix and a sequence's own pages.
// Where there are fewer units than the chip has room for, or a prefix, a
// segment is cut into splits that write partial results (unnormalised O, m, l)
// to the workspace, and a second launch adds them in split order.
//
//  * attn_stream: units of up to 32 rows (decode).  Bound by the read of K and
//    V: each wave streams keys of its own, 32 at a time, K straight into
//    operand registers, V through its own slice of LDS; nothing in the loop
//    waits for another wave.  Four sequences of 100 k to 131 k keys, 4 tokens
//    each: 357 us, 5.3 TB/s; 64 sequences of 1500 to 2500 keys 105 us, 4.8 TB/s.
//  * attn_tile: more rows (prompts, a shared prefix under many sequences).
//    Bound by the issue of MFMA and softmax instructions (per 32 rows x 64 keys
//    and wave 64 MFMAs, 1024 cycles, and about 200 others, 900 cycles, of which
//    two resident waves overlap half): four waves of 16 NQ rows share tiles of
//    64 keys in LDS, double-buffered.  Prompts of up to 7001 tokens over 9001
//    keys: 844 to 862 us, 1.0 PFLOP/s (one slower card: 932; a library product of
//    8192^3 runs at 1.20 to 1.22).
//
// Rounding: probabilities enter the second product as the cache's type, to
// nearest (off by 2^-8 of each at most in bf16, 2^-11 in fp16, and there by 2^-37
// of the row's largest where that is more; see kLift), beside the output's own
// rounding.  The second product then runs at the 16-bit rate.  Sums, maxima, O
// and the partial results are fp32, and l is summed from the unrounded
// probabilities.

#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Most splits of a call (the prefix's and a sequence's own together).
constexpr int kMaxSplits = 128;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <bool BF>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Probabilities are formed as 2^kLift of themselves.  fp16 keeps 11 bits of a
// number down to 2^-14 and none below 2^-25, so beside a row's largest (1; up to
// 2^3 in tiles, see kSlack) a long tail of small ones would lose its mass,
// always downward, while their sum l kept it.  2^12 keeps the largest below fp16's 65504 and
// moves that edge to 2^-37 of it.  The lift is taken off O and l together at
// the end of a unit, exactly, and takes no time (2048-token prompt 55.9 us without, 55.5
// with).  bf16 has the range of fp32.
template <bool BF>
constexpr float kLift = BF ? 0.f : 12.f;
template <bool BF>
constexpr float kUnlift = BF ? 1.f : 1.f / 4096.f;

// Two floats to two 16-bit values, round to nearest even (one instruction).
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), b16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}

// The two values of a lane pair (l, l ^ 32), then of the rows of 16 lanes.
// (Elements are copied out before they are reinterpreted: a bit cast of a
// vector's element takes element 0.)
__device__ __forceinline__ f32x2 swap32(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t x = r[0], y = r[1];
    return f32x2{__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
}

__device__ __forceinline__ f32x2 swap16(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t x = r[0], y = r[1];
    return f32x2{__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
}

// The larger value, NaN if either is (three operands an instruction; fmaxf
// would spend one more on each operand to quiet its NaN).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float larger(float t, const f32x4& v) {
    return larger(larger(larger(larger(t, v[0]), v[1]), v[2]), v[3]);
}

// Over the four lanes that share a row (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float v) {
    const f32x2 a = swap32(v);
    const f32x2 b = swap16(larger(a[0], a[1]));
    return larger(b[0], b[1]);
}

__device__ __forceinline__ float row_sum(float v) {
    const f32x2 a = swap32(v);
    const f32x2 b = swap16(a[0] + a[1]);
    return b[0] + b[1];
}

// How a call is cut; every field follows from the host's sizes alone.  A
// sequence's streamed unit has splits | 1 places in the grid: workgroups go to the four
// shader engines of an XCD in turn, and where sequences end early an even
// period would leave the same engines without work each time (16 sequences of
// 1 to 8192 keys 25.1 -> 23.6 us when it was changed).
struct Plan {
    int rows;              // most rows of a unit
    int blocks;            // row blocks of a unit
    int splits, len;       // of a sequence's own keys: splits of `len` keys
    int pblocks, psplits, plen;      // of the shared prefix, whose unit has every token's rows
    int pgrid;             // workgroups of the prefix, ahead of the others
    unsigned first;        // workgroup (of a join's kernels too) that the launch begins with
    int paired;            // order of the row blocks (see attn_tile)
    int direct;            // one split and no prefix: results go straight to out
    float* part;           // [psplits + splits][tokens * q_heads][dim], unnormalised
    float2* stat;          // [psplits + splits][tokens * q_heads]: m (in bits), l
};

// A row's place: its token (-1: none) and the keys it sees, [lo, hi) of the segment.
struct Row {
    int token, lo, hi;
};

// One unit's segment of keys.
struct Segment {
    const int32_t* table;
    int keys;              // keys of the segment
    int base;              // position of its first key
    Seq seq;               // of the sequence (own keys only)
};

__device__ __forceinline__ Row clip(const AttnArgs& a, int token, int pos, int keys, int base, int seg_keys) {
    Row r;
    r.token = token;
    const int hi = a.causal ? min(pos + 1, keys) : keys;
    const int lo = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
    r.hi = min(max(hi - base, 0), seg_keys);
    r.lo = min(max(lo - base, 0), seg_keys);
    return r;
}

template <bool PREFIX>
__device__ __forceinline__ Row row_place(const AttnArgs& a, const Segment& g, int row, int group) {
    const int i = row / group;
    if constexpr (!PREFIX) {
        if (i >= g.seq.count) return Row{-1, 0, 0};
        return clip(a, g.seq.start + i, g.seq.keys - g.seq.count + i, g.seq.keys, g.base, g.keys);
    }
    // the rows of every token: the last sequence that starts at or before it
    if (i >= a.batch.tokens) return Row{-1, 0, 0};
    int s = i / a.batch.q_len;
    if (a.batch.q_start) {
        s = -1;
        for (int j = 0; j < a.batch.num_seqs; ++j) s += a.batch.q_start[j] <= i;
        if (s < 0) return Row{-1, 0, 0};
    }
    const Seq q = load_seq(a.batch, s);
    if (i >= q.start + q.count) return Row{-1, 0, 0};
    return clip(a, i, q.keys - q.count + (i - q.start), q.keys, 0, g.keys);
}

// Row number in the pool of key `key` of the segment (a head's row of dim
// values), or -1 if its page is outside the pool.
__device__ __forceinline__ int pool_row(const AttnArgs& a, const Segment& g, int head, int key) {
    const int page = g.table[key >> a.cache.page_shift];
    const int in = key & ((1 << a.cache.page_shift) - 1);
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.cache.num_pages)) return -1;
    return ((page * a.cache.heads + head) << a.cache.page_shift) + in;
}

constexpr u32x4 kNaNs = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};   // NaN in fp16 and bf16
constexpr u32x4 kZeros = {0u, 0u, 0u, 0u};

// A block's queries as the second operand, with scale's sign: dims 32 i + 8 g ..
template <int D, bool BF>
__device__ __forceinline__ void load_q(const AttnArgs& a, const Row& r, int head, u32x4 (&q)[D / 32]) {
    const int g = (threadIdx.x & 63) >> 4;
    const uint16_t* p = a.q + static_cast<long long>(r.token) * a.q_stride + static_cast<long long>(head) * D + 8 * g;
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        q[i] = kZeros;
        if (r.token >= 0 && a.scale != 0.f) q[i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) q[i][j] ^= flip;
    }
}

// Running softmax of one row block over KB 16-key blocks of scores: s becomes
// probabilities (packed into p), m and l move on, o and l are rescaled if the
// maximum rose.  sc > 0 is |scale| log2 e; m is in the scores' own units; p, l and
// o carry the lift.
template <int KB, int ND, bool BF>
__device__ __forceinline__ void softmax_step(f32x4 (&s)[KB], uint32_t (&p)[KB][2], float sc, float& m, float& l,
                                             f32x4 (&o)[ND]) {
    float mx = m;
#pragma unroll
    for (int k = 0; k < KB; ++k) mx = larger(mx, s[k]);
    mx = row_max(mx);
    const float mc = mx == -INFINITY ? 0.f : mx * sc - kLift<BF>;
    if (__ballot(mx > m)) {
        const float old = m == -INFINITY ? mc : m * sc - kLift<BF>;
        const float c = __builtin_amdgcn_exp2f(old - mc);
        l *= c;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= c;
    }
    m = mx;
#pragma unroll
    for (int k = 0; k < KB; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[k][i] = __builtin_amdgcn_exp2f(fmaf(s[k][i], sc, -mc));
            l += s[k][i];
        }
        p[k][0] = pack2<BF>(s[k][0], s[k][1]);
        p[k][1] = pack2<BF>(s[k][2], s[k][3]);
    }
}

// Four neighbouring results to out.
__device__ __forceinline__ void store4(const AttnArgs& a, size_t at, f32x4 v) {
    if (a.out_dtype == DT_FP32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = v;
    } else {
        const u32x2 u = a.out_dtype == DT_BF16 ? u32x2{pack2<true>(v[0], v[1]), pack2<true>(v[2], v[3])}
                                               : u32x2{pack2<false>(v[0], v[1]), pack2<false>(v[2], v[3])};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = u;
    }
}

// Results of a row block (m in bits, l without the lift): o[d] holds dims
// 16 d + 4 g + 0..3 of the lane's row, with it.
template <int ND, bool BF>
__device__ __forceinline__ void finish(const AttnArgs& a, const Plan& pl, int slot, const Row& r, int head, float m,
                                       float l, const f32x4 (&o)[ND]) {
    if (r.token < 0) return;
    const int g = (threadIdx.x & 63) >> 4;
    constexpr int D = 16 * ND;
    const size_t row = static_cast<size_t>(r.token) * a.q_heads + head;
    if (!pl.direct) {
        const size_t at = static_cast<size_t>(slot) * a.batch.tokens * a.q_heads + row;
        float* to = pl.part + at * D + 4 * g;
#pragma unroll
        for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(to + 16 * d) = o[d] * kUnlift<BF>;
        if (g == 0) pl.stat[at] = float2{m, l};
        return;
    }
    const float inv = l != 0.f ? kUnlift<BF> / l : 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        store4(a, row * D + 16 * d + 4 * g, l != 0.f ? o[d] * inv : f32x4{0.f, 0.f, 0.f, 0.f});
    }
    if (a.lse && g == 0) a.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// V in LDS, row-major with D values a row, 16-byte chunk c of row r at place
// c ^ (r & kMask): rows of 128 bytes and more start on the same banks, the
// exclusive or spreads a column of rows over them.
template <int D>
__device__ __forceinline__ int swz(int row, int chunk) {
    constexpr int kMask = D / 8 < 16 ? D / 8 - 1 : 15;
    return row * (D / 8) + (chunk ^ (row & kMask));
}

// Operand of V^T: 16 dims (block d) x 32 keys (rows 32 kk ..) of a tile in LDS.
template <int D>
__device__ __forceinline__ u32x4 load_vt(const uint16_t* v, int kk, int d) {
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    u32x4 r;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int row = 32 * kk + 16 * half + 4 * g + (i >> 2);
        const int col = 16 * d + 4 * (i & 3);
        const uint16_t* p = v + 8 * swz<D>(row, col >> 3) + (col & 7);
        const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        const u32x2 u = __builtin_bit_cast(u32x2, t);
        r[2 * half] = u[0];
        r[2 * half + 1] = u[1];
    }
    return r;
}

// Values that are infinite or NaN.  0 times one of them is no zero, so where
// not every row sees every key of a tile, such values become zeros in LDS
// before the second product, and a pass over these tiles at the end adds them
// to the rows that see them (each is the whole result of its row and dim,
// whatever its probability).  Other tiles are not looked at, and the pass runs
// only where there were such values.
//
// The halves of a word whose exponent is all ones, as ones in bits 0 and 16.
template <bool BF>
__device__ __forceinline__ uint32_t not_finite(uint32_t v) {
    constexpr uint32_t kMask = BF ? 0x7f807f80u : 0x7c007c00u, kOne = BF ? 0x00800080u : 0x04000400u;
    return ((v & kMask) + kOne) >> 15 & 0x00010001u;
}

// v with such values as zeros; `bad` collects that there were some.
template <bool BF>
__device__ __forceinline__ u32x4 finite_or_zero(u32x4 v, uint32_t& bad) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t vi = v[i], b = not_finite<BF>(vi);
        v[i] = vi & ~((b << 16) - b);
        bad |= b;
    }
    return v;
}

// Of the `count` x 64 16-byte pieces from `at` (an even count), which this wave
// alone uses now.
template <bool BF>
__device__ __forceinline__ void clean_lds(uint32_t at, int count, uint32_t& bad) {
    at += 16 * (threadIdx.x & 63);
#pragma unroll 1
    for (int i = 0; i < count; i += 2, at += 2048) {
        lds_u32x4* const p = (lds_u32x4*)(uintptr_t)at;
        const u32x4 x = p[0], y = p[64];
        p[0] = finite_or_zero<BF>(x, bad);
        p[64] = finite_or_zero<BF>(y, bad);
    }
}

// The pass at the end for one row block over keys [from, to): o[d] holds dims
// 16 (first + d) + 4 g4 ..
template <int D, bool BF, int ND>
__device__ void add_not_finite(const AttnArgs& a, const Segment& seg, int head, const Row& row, int from, int to, int first,
                               f32x4 (&o)[ND]) {
    const int g4 = (threadIdx.x & 63) >> 4;
    for (int j = from; j < to; ++j) {
        const int r = pool_row(a, seg, head, j);
        if (r < 0) continue;
        const uint16_t* v = a.cache.v + static_cast<size_t>(r) * D + 16 * first + 4 * g4;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const u32x2 u = *reinterpret_cast<const u32x2*>(v + 16 * d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t ui = i & 2 ? u[1] : u[0];
                const uint16_t h = static_cast<uint16_t>(i & 1 ? ui >> 16 : ui);
                const float x = BF ? bf16_bits_to_f32(h) : f16_bits_to_f32(h);
                if (not_finite<BF>(h) && j >= row.lo && j < row.hi) o[d][i] += x;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

__device__ __forceinline__ Segment own_segment(const AttnArgs& a, int s) {
    Segment g;
    g.seq = load_seq(a.batch, s);
    g.table = a.batch.page_table + static_cast<size_t>(s) * a.batch.table_width;
    g.base = a.batch.prefix_len;
    g.keys = max(g.seq.keys - g.base, 0);
    return g;
}

__device__ __forceinline__ Segment prefix_segment(const AttnArgs& a) {
    return Segment{a.batch.prefix_table, min(a.batch.prefix_len, a.batch.key_limit), 0, Seq{0, 0, 0}};
}

// ------------------------------------------------------------- few rows

// Bytes of LDS: every wave's V, then the statistics and a flag of each.
constexpr int stream_lds(int D, int NQ) { return 256 * D + 512 * NQ + 16; }

//
// SAME: every row of a unit sees the same keys, [0, hi) (one token a sequence and
// no window), so only the last step has a mask and no value is hidden from a row
// that its neighbours see.  Keys from hi on, which there are where a sequence
// has more new tokens than are attended for, are taken as past the end.
template <int D, bool BF, int NQ, bool PREFIX, bool SAME>
__device__ __forceinline__ void attn_stream(const AttnArgs& a, const Plan& pl, int id, unsigned char* lds) {
    constexpr int NS = D / 32, ND = D / 16, CH = D / 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g4 = lane >> 4, col = lane & 15;
    uint16_t* const vl = reinterpret_cast<uint16_t*>(lds) + wave * 32 * D;
    float2(*stat)[16 * NQ] = reinterpret_cast<float2(*)[16 * NQ]>(lds + 256 * D);
    const int Hk = a.cache.heads, group = a.q_heads / Hk;
    const int head = id % Hk;
    int rest = id / Hk;
    const int splits = PREFIX ? pl.psplits : pl.splits, len = PREFIX ? pl.plen : pl.len;
    const int places = PREFIX ? splits : splits | 1;  // see Plan
    const int split = rest % places;
    rest /= places;
    if (split >= splits) return;
    const int begin = split * len;
    // the first step's pages, looked up beside the lengths (entries are in
    // bounds up to the host's limit; what stands behind a length is not used)
    int first = -2;
    if (a.window == 0) {
        const Segment any = PREFIX ? prefix_segment(a)
                                   : Segment{a.batch.page_table + static_cast<size_t>(rest) * a.batch.table_width,
                                             a.batch.key_limit - a.batch.prefix_len, 0, Seq{0, 0, 0}};
        const int key = begin + 32 * wave + (lane & 31);
        if (key < any.keys) first = pool_row(a, any, head, key);
    }
    const Segment seg = PREFIX ? prefix_segment(a) : own_segment(a, rest);
    const int end = min(begin + len, seg.keys);
    if (begin >= end && !pl.direct) return;

    Row row[NQ];
    u32x4 q[NQ][NS];
    int hidx[NQ];
    int lo = 0x7fffffff, hi = 0, full_lo = 0, full_hi = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = 16 * n + col;
        row[n] = r < (PREFIX ? a.batch.tokens * group : pl.rows) ? row_place<PREFIX>(a, seg, r, group) : Row{-1, 0, 0};
        hidx[n] = head * group + r % group;
        load_q<D, BF>(a, row[n], hidx[n], q[n]);
        if (row[n].hi > row[n].lo) lo = min(lo, row[n].lo), hi = max(hi, row[n].hi);
        if (row[n].token >= 0) full_lo = max(full_lo, row[n].lo), full_hi = min(full_hi, row[n].hi);
    }
    // the wave's steps cover the keys that any of its rows sees; between full_lo
    // and full_hi every row sees them all
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
        lo = min(lo, __shfl_xor(lo, off, 64));
        hi = max(hi, __shfl_xor(hi, off, 64));
        full_lo = max(full_lo, __shfl_xor(full_lo, off, 64));
        full_hi = min(full_hi, __shfl_xor(full_hi, off, 64));
    }
    full_lo = __builtin_amdgcn_readfirstlane(full_lo);
    full_hi = __builtin_amdgcn_readfirstlane(full_hi);
    lo = max(lo, begin) & ~31;
    hi = min(hi, end);
    if (hi <= lo) lo = hi = 0;                        // nothing to see here
    const float sc = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;

    float m[NQ], l[NQ];
    f32x4 o[NQ][ND];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kr[2][NS], vr[CH / 2];
    constexpr int VR = CH / 2;                // 32 rows x CH chunks over 64 lanes
    // lane l looks up key l of a step; the lanes that load a row ask for it
    const int there = SAME ? hi : seg.keys;
    const auto look = [&](int at) { return at + (lane & 31) < there ? pool_row(a, seg, head, at + (lane & 31)) : -2; };
    const auto fetch = [&](int where) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int r = __shfl(where, 16 * b + col, 64);
            const uint16_t* p = a.cache.k + static_cast<size_t>(r < 0 ? 0 : r) * D + 8 * g4;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                kr[b][i] = r == -1 ? kNaNs : kZeros;
                if (r >= 0) kr[b][i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
            }
        }
#pragma unroll
        for (int i = 0; i < VR; ++i) {
            const int c = lane + 64 * i;
            const int r = __shfl(where, c / CH, 64);
            vr[i] = kZeros;
            if (r >= 0) vr[i] = *reinterpret_cast<const u32x4*>(a.cache.v + static_cast<size_t>(r) * D + 8 * (c % CH));
        }
    };

    const auto masked = [&](int step) { return step < full_lo || min(step + 32, seg.keys) > full_hi; };
    const uint32_t vat = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte*)vl));
    uint32_t unseen = 0;
    int at = lo + 32 * wave;
    if (at < hi) {
        // without a window the first step is the one looked up above
        if (a.window == 0) fetch(at + (lane & 31) < there ? first : -2);
        else fetch(look(at));
        int next = look(at + 128);
        for (; at < hi; at += 128) {
            f32x4 s[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    s[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < NS; ++i) s[n][b] = mma<BF>(kr[b][i], q[n][i], s[n][b]);
                }
#pragma unroll
            for (int i = 0; i < VR; ++i) {
                const int c = lane + 64 * i;
                *reinterpret_cast<u32x4*>(vl + 8 * swz<D>(c / CH, c % CH)) = vr[i];
            }
            if (!SAME && masked(at)) clean_lds<BF>(vat, VR, unseen);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int cur = at;
            if (at + 128 < hi) {
                fetch(next);
                next = look(at + 256);
            }
            uint32_t p[NQ][2][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                if (!SAME || cur + 32 > hi) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = cur + 16 * b + 4 * g4 + i;
                            if ((!SAME && key < row[n].lo) || key >= (SAME ? hi : min(row[n].hi, end))) s[n][b][i] = -INFINITY;
                        }
                }
                softmax_step<2, ND, BF>(s[n], p[n], sc, m[n], l[n], o[n]);
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const u32x4 vt = load_vt<D>(vl, 0, d);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    o[n][d] = mma<BF>(vt, u32x4{p[n][0][0], p[n][0][1], p[n][1][0], p[n][1][1]}, o[n][d]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }

    // the four waves' results meet: maxima first, then the rescaled sums, in
    // wave order, through the V buffers (16 NQ rows x D floats)
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        l[n] = row_sum(l[n]);
        if (g4 == 0) stat[wave][16 * n + col] = float2{m[n], l[n]};
    }
    uint32_t* const unclean = reinterpret_cast<uint32_t*>(lds + 256 * D + 512 * NQ);
    const bool mine = __ballot(unseen) != 0;
    if (lane == 0) unclean[wave] = mine;
    __syncthreads();
    const bool dirty = (unclean[0] | unclean[1] | unclean[2] | unclean[3]) != 0;
    float* const sum = reinterpret_cast<float*>(lds);     // one row block of every wave
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) mm = fmaxf(mm, stat[w][16 * n + col].x);
        // what the lifted sums are multiples of: the exponent that softmax_step took off
        const auto taken = [&](float t) { return t * sc - kLift<BF>; };
        const float mc = mm == -INFINITY ? 0.f : taken(mm);
        const float top = mm == -INFINITY ? -INFINITY : mc + kLift<BF>;
        float ll = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 t = stat[w][16 * n + col];
            if (t.x != -INFINITY || t.y != 0.f) ll += t.y * __builtin_amdgcn_exp2f((t.x == -INFINITY ? mc : taken(t.x)) - mc);
        }
        ll *= kUnlift<BF>;
        const float c = __builtin_amdgcn_exp2f((m[n] == -INFINITY ? mc : taken(m[n])) - mc) * kUnlift<BF>;
        if (n) __syncthreads();
#pragma unroll
        for (int d = 0; d < ND; ++d)
            *reinterpret_cast<f32x4*>(sum + (wave * 16 + col) * D + 4 * ((4 * d + g4) ^ col)) = o[n][d] * c;
        __syncthreads();
        // wave w adds the quarter of the dims it stores
        constexpr int PER = ND / 4;
        f32x4 r[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            r[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w)
                r[j] += *reinterpret_cast<const f32x4*>(sum + (w * 16 + col) * D + 4 * ((4 * (wave * PER + j) + g4) ^ col));
        }
        if (!SAME && dirty)
            for (int step = lo; step < hi; step += 32)
                if (masked(step)) add_not_finite<D, BF>(a, seg, head, row[n], step, min(step + 32, hi), wave * PER, r);
        if (row[n].token < 0) continue;
        const size_t rw = static_cast<size_t>(row[n].token) * a.q_heads + hidx[n];
        const int slot = PREFIX ? split : pl.psplits + split;
        if (!pl.direct) {
            const size_t at2 = static_cast<size_t>(slot) * a.batch.tokens * a.q_heads + rw;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                *reinterpret_cast<f32x4*>(pl.part + at2 * D + 16 * (wave * PER + j) + 4 * g4) = r[j];
            if (g4 == 0 && wave == 0) pl.stat[at2] = float2{top, ll};
        } else {
            const float inv = ll != 0.f ? 1.0f / ll : 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                store4(a, rw * D + 16 * (wave * PER + j) + 4 * g4, ll != 0.f ? r[j] * inv : f32x4{0.f, 0.f, 0.f, 0.f});
            }
            if (a.lse && g4 == 0 && wave == 0)
                a.lse[rw] = ll != 0.f ? (top + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
        }
    }
}

// ------------------------------------------------------------- many rows

// What a lane copies for a key that is not there: zeros for one past the
// segment, NaN for one whose page is outside the pool.
__device__ const u32x4 absent[2] = {{0u, 0u, 0u, 0u}, {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu}};

// 64 x 16 bytes from global memory straight to LDS at `to` (the same for the
// whole wave), in lane order.  Written as assembly, which returns no register:
// the compiler, which cannot tell the two halves of a double buffer apart,
// would wait for these copies before every later LDS read.  copies_done()
// waits for them.
__device__ __forceinline__ void copy_to_lds(uint32_t to, const void* base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds(uint32_t to, const void* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A value that is the same for the whole wave, by a scalar load (read-only
// memory during the kernel), which does not queue behind the copies.
__device__ __forceinline__ int load_scalar(const int32_t* p) {
    return *(const __attribute__((address_space(4))) int32_t*)p;
}

// Keys of a tile: 64, or 32 for 256-wide heads (two workgroups' tiles fit a CU).
constexpr int tile_keys(int D) { return D > 128 ? 32 : 64; }

// A step of the loop needs V of tile i and K of tile i + 1: the scores of the
// next tile are multiplied while this one's become probabilities, so the
// matrix and vector units of a SIMD both have work of one wave.  K and V have
// two buffers each, filled by direct copies to LDS that are issued a step
// ahead.  A maximum within 2^kSlack of the one in use leaves it in use
// (probabilities up to 2^kSlack; every result divides by their sum), which
// saves nearly all rescaling but rounds a row's largest probability, that a
// current maximum makes exactly 1.  With a slack of 0, 3 and 6 ragged prompts
// take 879, 845 and 833 us, and their error against 64 bits is 1.10, 1.16 and
// 1.26 times that of one final rounding.
constexpr float kSlack = 3.f;

//
// Blocks are numbered from the last row down: causal rows see more keys the
// later they stand, and the longest should start first.  Where all workgroups
// are resident at once (`paired`) the lower half counts up again instead: the
// second workgroup on a CU is then short where the first is long (2048-token
// prompt 57.5 -> 54.9 us).  Sequences vary slowest: workgroups go to the shader
// engines in turn, so a sequence without rows at every fourth place would leave
// an engine idle (ragged prompts 858 -> 2122 us that way round).
constexpr int tile_lds(int D) { return 4 * tile_keys(D) * D * 2; }

template <int D, bool BF, int NQ, bool PREFIX>
__device__ __forceinline__ void attn_tile(const AttnArgs& a, const Plan& pl, int id, unsigned char* lds) {
    constexpr int NS = D / 32, ND = D / 16, CH = D / 8, KT = tile_keys(D), KB = KT / 16;
    constexpr int RW = 64 * NQ;                       // rows of a workgroup
    constexpr int WR = KT / 4;                        // keys of a tile that a wave copies
    constexpr int CP = WR * CH / 64;                  // copies of 64 x 16 bytes a wave makes
    constexpr int TILE = KT * D * 2;                  // bytes
    unsigned char* const tiles = lds;                 // K0, V0, K1, V1
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g4 = lane >> 4, col = lane & 15;
    const int Hk = a.cache.heads, group = a.q_heads / Hk;
    const int head = id % Hk;
    int rest = id / Hk;
    const int splits = PREFIX ? pl.psplits : pl.splits, len = PREFIX ? pl.plen : pl.len;
    const int split = rest % splits;
    rest /= splits;
    const int blocks = PREFIX ? pl.pblocks : pl.blocks, upper = (blocks + 1) / 2, nth = rest % blocks;
    const int block = pl.paired && nth >= upper ? nth - upper : blocks - 1 - nth;
    const Segment seg = PREFIX ? prefix_segment(a) : own_segment(a, rest / blocks);
    const int nrows = (PREFIX ? a.batch.tokens : min(seg.seq.count, a.batch.q_len)) * group;
    if (block * RW >= nrows) return;
    const int begin = split * len, end = min(begin + len, seg.keys);
    if (begin >= end && !pl.direct) return;

    Row row[NQ];
    u32x4 q[NQ][NS];
    int hidx[NQ];
    int lo = 0x7fffffff, hi = 0, full_lo = 0, full_hi = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = block * RW + wave * 16 * NQ + 16 * n + col;
        row[n] = r < nrows ? row_place<PREFIX>(a, seg, r, group) : Row{-1, 0, 0};
        row[n].hi = max(min(row[n].hi, end), row[n].lo);
        hidx[n] = head * group + r % group;
        load_q<D, BF>(a, row[n], hidx[n], q[n]);
        if (row[n].hi > row[n].lo) lo = min(lo, row[n].lo), hi = max(hi, row[n].hi);
        if (row[n].token >= 0) full_lo = max(full_lo, row[n].lo), full_hi = min(full_hi, row[n].hi);
    }
    // the wave's bounds (tiles it works on, tiles without a mask), then the workgroup's
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
        lo = min(lo, __shfl_xor(lo, off, 64));
        hi = max(hi, __shfl_xor(hi, off, 64));
        full_lo = max(full_lo, __shfl_xor(full_lo, off, 64));
        full_hi = min(full_hi, __shfl_xor(full_hi, off, 64));
    }
    int(*bounds)[4] = reinterpret_cast<int(*)[4]>(lds);         // ahead of the first tile and behind the last
    if (lane == 0) bounds[0][wave] = lo, bounds[1][wave] = hi, bounds[2][wave] = full_lo, bounds[3][wave] = full_hi;
    __syncthreads();
    const int wlo = __builtin_amdgcn_readfirstlane(lo), whi = __builtin_amdgcn_readfirstlane(hi);
    int all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lo = min(lo, bounds[0][w]);
        hi = max(hi, bounds[1][w]);
        all_lo = max(all_lo, bounds[2][w]);
        all_hi = min(all_hi, bounds[3][w]);
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    __syncthreads();
    lo = __builtin_amdgcn_readfirstlane(max(lo, begin) & ~(KT - 1));
    hi = __builtin_amdgcn_readfirstlane(hi);
    full_lo = __builtin_amdgcn_readfirstlane(full_lo);
    full_hi = __builtin_amdgcn_readfirstlane(full_hi);
    const float sc = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;

    float m[NQ], mc[NQ], l[NQ];                       // mc = m sc - lift, 0 before any key
    f32x4 o[NQ][ND], s[NQ][KB];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY;
        mc[n] = l[n] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Copies: the wave's keys WR wave .. of a tile; LDS place c ^ row & mask
    // holds chunk c, so the lanes of a copy (places in order) ask for the
    // chunks that belong there.
    uint32_t from[CP];
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const int c = 64 * i + lane, r = c / CH;
        from[i] = (r * D + 8 * (swz<D>(WR * wave + r, c % CH) % CH)) * 2;
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte*)tiles));
    const bool paged = (1 << a.cache.page_shift) >= WR;         // a wave's keys of a tile lie in one page
    const auto page_of = [&](int at) {
        const int key = at + WR * wave;
        return paged && key < seg.keys ? load_scalar(seg.table + (key >> a.cache.page_shift)) : -1;
    };
    const auto copy = [&](const uint16_t* pool, uint32_t to, int at, int page) {
        to += WR * wave * D * 2;
        if (static_cast<unsigned>(page) < static_cast<unsigned>(a.cache.num_pages) && at + KT <= seg.keys) {
            const int in = (at + WR * wave) & ((1 << a.cache.page_shift) - 1);
            const uint16_t* src = pool + static_cast<size_t>(((page * Hk + head) << a.cache.page_shift) + in) * D;
#pragma unroll
            for (int i = 0; i < CP; ++i) copy_to_lds(to + 1024 * i, src, from[i]);
        } else {
#pragma unroll
            for (int i = 0; i < CP; ++i) {
                const int key = at + WR * wave + (64 * i + lane) / CH;
                const int r = key < seg.keys ? pool_row(a, seg, head, key) : -2;
                const char* src = r >= 0 ? reinterpret_cast<const char*>(pool + static_cast<size_t>(r) * D) +
                                               from[i] % (2 * D)
                                         : reinterpret_cast<const char*>(&absent[r + 2]);
                copy_to_lds(to + 1024 * i, src);
            }
        }
    };

    // LDS addresses of the wave's reads: of K, row 16 b + col, chunk 4 i + g4; of
    // V^T, rows 32 kk + 16 half + 4 g4 + (col >> 2), columns 16 d + 4 (col & 3)
    uint32_t kat[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) kat[i] = 16 * swz<D>(col, 4 * i + g4);
    const int vrow = 4 * g4 + (col >> 2);
    const uint32_t vat = 16 * swz<D>(vrow, (col & 3) >> 1) + 8 * (col & 1);

    const auto scores = [&](uint32_t kt) {
#pragma unroll
        for (int b = 0; b < KB; ++b) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const u32x4 kf = *(const lds_u32x4*)((const lds_byte*)(uintptr_t)(kt + kat[i]) + 32 * D * b);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][b] = mma<BF>(kf, q[n][i], s[n][b]);
            }
        }
    };
    // a row's largest score of the tile in s: `values` finds it for the next
    // tile between its MFMAs, a masked tile and the first one find it here
    float mx[NQ];
    const auto find_top = [&]() {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            mx[n] = -INFINITY;
#pragma unroll
            for (int b = 0; b < KB; ++b) mx[n] = larger(mx[n], s[n][b]);
            mx[n] = row_max(mx[n]);
        }
    };
    const auto masked = [&](int at) { return at < full_lo || at + KT > full_hi; };
    const auto hides = [&](int at) { return at < all_lo || min(at + KT, seg.keys) > all_hi; };     // of the workgroup's rows
    uint32_t unseen = 0;
    // masks and, where a maximum rose past the slack, the new reference
    const auto settle = [&](int at) {
        if (masked(at)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // lo <= key < hi
                        const unsigned past = at + 16 * b + 4 * g4 + i - row[n].lo;
                        if (past >= static_cast<unsigned>(row[n].hi - row[n].lo)) s[n][b][i] = -INFINITY;
                    }
            find_top();
        }
        bool rose = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            rose |= m[n] == -INFINITY ? mx[n] != -INFINITY : mx[n] * sc > mc[n] + (kLift<BF> + kSlack);
        if (__ballot(rose)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const float top = fmaxf(mx[n], m[n]);
                const float now = top == -INFINITY ? 0.f : top * sc - kLift<BF>;
                const float c = m[n] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mc[n] - now);
                m[n] = top;
                mc[n] = now;
                l[n] *= c;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[n][d] *= c;
            }
        }
    };
    // this tile's scores to probabilities, block by block, each block's place
    // taken by the next tile's scores as it becomes free (behind the last tile
    // they are of whatever the buffer holds, and nothing uses them).  LDS is
    // read ahead of its use: K a block of 16 keys, V^T kAhead operands, since a
    // wave that waits for each read leaves both units idle; the scheduling
    // barriers keep the compiler from sinking the reads to their uses.
    constexpr int kAhead = 4, VF = KB / 2 * ND;
    u32x4 kf[2][NS], vf[kAhead];
    const auto read_k = [&](u32x4 (&f)[NS], uint32_t kt, int b) {
#pragma unroll
        for (int i = 0; i < NS; ++i) f[i] = *(const lds_u32x4*)((const lds_byte*)(uintptr_t)(kt + kat[i]) + 32 * D * b);
    };
    const auto read_v = [&](uint32_t vt, int n) {
        lds_byte* at = (lds_byte*)(uintptr_t)(vt + (vat ^ (32 * (n % ND)))) + 64 * D * (n / ND);
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 32 * D));
        const u32x2 ux = __builtin_bit_cast(u32x2, x), uy = __builtin_bit_cast(u32x2, y);
        return u32x4{ux[0], ux[1], uy[0], uy[1]};
    };
    const auto turn = [&](uint32_t (&p)[NQ][KB][2], uint32_t kt, uint32_t vt, auto between) {
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            if (b + 1 < KB) {
                read_k(kf[(b + 1) & 1], kt, b + 1);
            } else {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) vf[i] = read_v(vt, i);
            }
            f32x4 to[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) to[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int n = 0; n < NQ; ++n) to[n] = mma<BF>(kf[b & 1][i], q[n][i], to[n]);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][b][i] = __builtin_amdgcn_exp2f(fmaf(s[n][b][i], sc, -mc[n]));
                    l[n] += s[n][b][i];
                }
                p[n][b][0] = pack2<BF>(s[n][b][0], s[n][b][1]);
                p[n][b][1] = pack2<BF>(s[n][b][2], s[n][b][3]);
                s[n][b] = to[n];
            }
            __builtin_amdgcn_sched_barrier(0);
            between(b);
        }
    };
    const auto values = [&](const uint32_t (&p)[NQ][KB][2], uint32_t vt) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) mx[n] = -INFINITY;
#pragma unroll
        for (int i = 0; i < VF; ++i) {
            const int kk = i / ND, d = i % ND;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
                o[n][d] = mma<BF>(vf[i % kAhead], u32x4{p[n][2 * kk][0], p[n][2 * kk][1], p[n][2 * kk + 1][0], p[n][2 * kk + 1][1]},
                                  o[n][d]);
            if (i + kAhead < VF) vf[i % kAhead] = read_v(vt, i + kAhead);
            // blocks of the next tile's scores, spread over the first half
            constexpr int AT = VF / 2 >= KB ? VF / 2 / KB : 1;
            if (i % AT == 0 && i / AT < KB) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) mx[n] = larger(mx[n], s[n][i / AT]);
            }
            if (i == VF - VF / 4) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) mx[n] = row_max(mx[n]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (lo < hi) {
        const auto mine = [&](int at) { return at < whi && at + KT > wlo; };
        int page_v = page_of(lo), page_k = page_of(lo + KT);
        copy(a.cache.k, base, lo, page_v);
        copies_done();
        __syncthreads();
        copy(a.cache.v, base + TILE, lo, page_v);
        if (lo + KT < hi) copy(a.cache.k, base + 2 * TILE, lo + KT, page_k);
        page_v = page_k;
        page_k = page_of(lo + 2 * KT);
        if (mine(lo)) {
            scores(base);
            find_top();
        }
        int buf = 0;
        for (int at = lo; at < hi; at += KT, buf ^= 1) {
            copies_done();
            if (hides(at)) clean_lds<BF>(base + (2 * buf + 1) * TILE + WR * wave * D * 2, CP, unseen);
            __syncthreads();              // V of this tile and K of the next are there, their other buffers free
            const uint32_t kt = base + 2 * (buf ^ 1) * TILE, vt = base + (2 * buf + 1) * TILE;
            const auto copy_next = [&](int what) {
                if (what == 0 && at + KT < hi) copy(a.cache.v, base + (2 * (buf ^ 1) + 1) * TILE, at + KT, page_v);
                if (what == 1) {
                    if (at + 2 * KT < hi) copy(a.cache.k, base + 2 * buf * TILE, at + 2 * KT, page_k);
                    page_v = page_k;
                    page_k = page_of(at + 3 * KT);
                }
            };
            if (mine(at)) {
                read_k(kf[0], kt, 0);
                settle(at);
                uint32_t p[NQ][KB][2];
                turn(p, kt, vt, copy_next);
                values(p, vt);
            } else {
                copy_next(0);
                copy_next(1);
                if (mine(at + KT)) {
                    scores(kt);
                    find_top();
                }
            }
        }
    }
    const bool found = __ballot(unseen) != 0;
    __syncthreads();
    if (lane == 0) bounds[0][wave] = found;
    __syncthreads();
    const bool dirty = (bounds[0][0] | bounds[0][1] | bounds[0][2] | bounds[0][3]) != 0;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if (dirty)
            for (int at = lo; at < hi; at += KT)
                if (hides(at)) add_not_finite<D, BF>(a, seg, head, row[n], at, min(at + KT, hi), 0, o[n]);
        finish<ND, BF>(a, pl, PREFIX ? split : pl.psplits + split, row[n], hidx[n], m[n] == -INFINITY ? -INFINITY : mc[n] + kLift<BF>,
                       row_sum(l[n]) * kUnlift<BF>, o[n]);
    }
}

// The same for many rows of few splits: D / 4 lanes a row, the splits in turn,
// so a workgroup finishes 256 / (D / 4) rows (32000 rows of 2 splits take 12 us
// so, 33 with a workgroup each).
constexpr int kRowSplits = 8;

template <int D>
__global__ __launch_bounds__(256) void attn_join_rows_kernel(AttnArgs a, Plan pl) {
    constexpr int LANES = D / 4, AT = 256 / LANES;
    const size_t rows = static_cast<size_t>(a.batch.tokens) * a.q_heads;
    const size_t row = static_cast<size_t>(pl.first + blockIdx.x) * AT + threadIdx.x / LANES;
    const int at = threadIdx.x % LANES, total = pl.psplits + pl.splits;
    if (row >= rows) return;
    float2 st[kRowSplits];
    f32x4 v[kRowSplits];
#pragma unroll
    for (int i = 0; i < kRowSplits; ++i)
        if (i < total) {
            st[i] = pl.stat[i * rows + row];
            v[i] = reinterpret_cast<const f32x4*>(pl.part + (i * rows + row) * D)[at];
        }
    // the row's sequence: a scan of the starts by every lane (rows of a wave
    // belong to different tokens)
    const int t = static_cast<int>(row / a.q_heads);
    int s = t / a.batch.q_len;
    if (a.batch.q_start) {
        s = -1;
        for (int j = 0; j < a.batch.num_seqs; ++j) s += a.batch.q_start[j] <= t;
        if (s < 0) return;
    }
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count || t - q.start >= a.batch.q_len) return;
    const int live = pl.psplits + (max(q.keys - a.batch.prefix_len, 0) + pl.len - 1) / pl.len;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kRowSplits; ++i)
        if (i < live) m = fmaxf(m, st[i].x);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kRowSplits; ++i)
        if (i < live && st[i].y != 0.f) {
            const float w = __builtin_amdgcn_exp2f((st[i].x == -INFINITY ? base : st[i].x) - base);
            l += w * st[i].y;
            acc += v[i] * w;
        }
    const float inv = l != 0.f ? 1.0f / l : 0.f;
    store4(a, row * D + 4 * at, l != 0.f ? acc * inv : f32x4{0.f, 0.f, 0.f, 0.f});
    if (a.lse && at == 0) a.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------- one launch

// How a segment's units are worked: not at all, streamed (16 or 32 rows, S0 of
// 16 that all see the same keys) or by tiles (64 or 128 rows a workgroup).
enum { NONE = 0, S1 = 1, S2 = 2, T1 = 3, T2 = 4, S0 = 5 };

constexpr int lds_bytes(int D, int kind) {
    return kind == NONE ? 0 : kind == S0 ? stream_lds(D, 1) : kind <= S2 ? stream_lds(D, kind) : tile_lds(D);
}

// The prefix's and the sequences' own workgroups side by side, so the tiles of
// the one and the streams of the other share the CUs.  Streams of 16 rows fit
// three workgroups on a CU (168 registers), streams of 256-wide heads one (367;
// held to 256 they spill: 16 sequences of 200 to 8000 keys 266 against 78 us),
// the rest two.
template <int D, bool BF, int P, int O>
__global__ __launch_bounds__(256, (O <= S2 || O == S0) && D > 128 ? 1 : P == NONE && O == S0 ? 3 : 2) void attn_kernel(
    AttnArgs a, Plan pl) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int id = static_cast<int>(pl.first + blockIdx.x);
    if constexpr (P != NONE) {
        if (id < pl.pgrid) {
            if constexpr (P <= S2) attn_stream<D, BF, P, true, false>(a, pl, id, lds);
            else attn_tile<D, BF, P - S2, true>(a, pl, id, lds);
            return;
        }
    }
    if constexpr (O == S0) attn_stream<D, BF, 1, false, true>(a, pl, id - pl.pgrid, lds);
    else if constexpr (O <= S2) attn_stream<D, BF, O, false, false>(a, pl, id - pl.pgrid, lds);
    else attn_tile<D, BF, O - S2, false>(a, pl, id - pl.pgrid, lds);
}

// ------------------------------------------------------------- joining splits

// Bound by its chain of reads (length and statistics, then the parts): 32 rows
// of 17 splits 4 us, 2048 of 20 6 us.
// One workgroup a row: sum_i w_i O_i / sum_i w_i l_i, w_i = 2^{m_i - max m},
// over the row's live splits.  Splits that hold no key of the row's sequence
// were never written and are not used.  256 / (D / 4) splits are read at a
// time, 16 bytes a lane; partial sums over a lane's splits meet in LDS, so the
// order of the additions depends on the number of splits alone.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, Plan pl) {
    constexpr int LANES = D / 4, AT = 256 / LANES;
    __shared__ float weight[kMaxSplits];
    __shared__ f32x4 sums[AT][LANES];
    const int tid = threadIdx.x, lane = tid & 63;
    const size_t rows = static_cast<size_t>(a.batch.tokens) * a.q_heads;
    const size_t row = pl.first + blockIdx.x;
    const int t = static_cast<int>(row / a.q_heads);
    const int total = pl.psplits + pl.splits;
    // the statistics of every split, read ahead of the length that says which count
    float2 st[kMaxSplits / 64];
#pragma unroll
    for (int j = 0; j < kMaxSplits / 64; ++j) {
        st[j] = float2{-INFINITY, 0.f};
        if (64 * j < total && 64 * j + lane < total) st[j] = pl.stat[(64 * j + lane) * rows + row];
    }
    const int s = seq_of(a.batch, t);
    if (s < 0) return;
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count || t - q.start >= a.batch.q_len) return;
    const int own = max(q.keys - a.batch.prefix_len, 0);
    const int live = pl.psplits + (own + pl.len - 1) / pl.len;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kMaxSplits / 64; ++j)
        if (64 * j + lane < live) m = fmaxf(m, st[j].x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int j = 0; j < kMaxSplits / 64; ++j)
        if (64 * j < live) {
            // l = 0: no key seen there, whatever its sums hold (weight -1); a
            // weight that is 0 itself still counts, as sums may be infinite
            const bool used = 64 * j + lane < live && st[j].y != 0.f;
            const float w = used ? __builtin_amdgcn_exp2f((st[j].x == -INFINITY ? base : st[j].x) - base) : -1.f;
            if (tid < 64) weight[64 * j + lane] = w;
            l += used ? w * st[j].y : 0.f;
        }
    l = wave_sum(l);
    __syncthreads();
    const int part = tid / LANES, at = tid % LANES;
    const f32x4* from = reinterpret_cast<const f32x4*>(pl.part + row * D) + at;
    const size_t step = rows * (D / 4);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = part; i < live; i += AT) {
        const float w = weight[i];
        const f32x4 v = from[i * step];
        if (w != -1.f) acc += v * w;
    }
    sums[part][at] = acc;
    __syncthreads();
    if (tid >= LANES) return;
    acc = sums[0][at];
#pragma unroll
    for (int j = 1; j < AT; ++j) acc += sums[j][at];
    const float inv = l != 0.f ? 1.0f / l : 0.f;
    store4(a, row * D + 4 * at, l != 0.f ? acc * inv : f32x4{0.f, 0.f, 0.f, 0.f});
    if (a.lse && tid == 0) a.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

// Rows up to which a unit streams, and rows of a tile workgroup.  Heads of 256
// keep to one row block a wave: two do not fit 256 registers beside the sums.
int stream_rows(int dim) { return dim > 128 ? 16 : 32; }

// 64 rows to a tile workgroup where 128 would leave half the CUs without one
// (a 300-token prompt 14.5 -> 11.1 us, 256 tokens over 4096 keys 39.2 -> 36.6);
// otherwise 128: each LDS read then feeds two MFMAs (2048 tokens over 4096 keys
// 138 against 174 us).
int tile_rows(const KvCache& c, const KvBatch& b, long long rows) {
    return c.dim > 128 || ((rows + 127) / 128) * b.num_seqs * c.heads < 128 ? 64 : 128;
}

// Splits of `keys` keys for `units` workgroups without splitting: enough to
// give the chip `want` workgroups, none under `least` keys.
void cut(long long units, int keys, int want, int least, int* splits, int* len) {
    int n = ceil_div(want, units);
    const int most = keys > least ? ceil_div(keys, least) : 1;
    if (n > most) n = most;
    if (n > kMaxSplits / 2) n = kMaxSplits / 2;
    if (n < 1) n = 1;
    *len = keys > 0 ? ceil_div(ceil_div(keys, n), least) * least : least;
    *splits = keys > 0 ? ceil_div(keys, *len) : 1;
}

int kind_of(const KvCache& c, const KvBatch& b, long long rows) {
    return rows <= 16 ? S1 : rows <= stream_rows(c.dim) ? S2 : tile_rows(c, b, rows) == 64 ? T1 : T2;
}

Plan make_plan(const KvCache& c, const KvBatch& b, int q_heads) {
    Plan p{};
    const int group = q_heads / c.heads;
    const long long rows = static_cast<long long>(b.q_len) * group;
    p.rows = static_cast<int>(rows);
    const int own = b.key_limit > b.prefix_len ? b.key_limit - b.prefix_len : 0;
    const bool stream = rows <= stream_rows(c.dim);
    p.blocks = stream ? 1 : ceil_div(rows, tile_rows(c, b, rows));
    const long long units = static_cast<long long>(b.num_seqs) * c.heads * p.blocks;
    // Streams: splits of at least 128 keys, one step of each wave, while units
    // are few; 256 from 256 units on (64 under a prefix 38.8 -> 37.1 us, where
    // one sequence of 2049 keys would take 12.2 for 10.7), and then one split
    // without a join up to 512 keys (64 sequences of 10 to 300 keys 14.8 -> 11.0
    // us; one of 500 would take 11.8 for 9.9).  4096 workgroups in all where
    // three fit a CU (16 ragged sequences 23.0 us, 25.7 with 2048), else 2048
    // (256-wide heads 88 -> 78 us, 24 rows a unit 53 -> 49).
    const bool many = units >= 256;
    const int least = !many ? 128 : own <= 512 && b.prefix_len == 0 ? 512 : 256;
    const int want = rows <= 16 && c.dim <= 128 ? 4096 : 2048;
    // Tiles: whole while every CU has a unit (1000-token prompt 29.8 us, 43.6 in
    // two splits), else two workgroups a CU (500 tokens over 6000 keys 72.6 us,
    // 82.0 with one a CU).
    cut(units, own, stream ? want : many ? 256 : 512, stream ? least : 512, &p.splits, &p.len);
    p.paired = units * p.splits <= 512;
    const int keys = b.prefix_len < b.key_limit ? b.prefix_len : b.key_limit;
    if (keys > 0) {
        const long long prows = static_cast<long long>(b.tokens) * group;
        const bool ps = prows <= stream_rows(c.dim);
        p.pblocks = ps ? 1 : ceil_div(prows, c.dim > 128 ? 64 : 128);
        cut(static_cast<long long>(c.heads) * p.pblocks, keys, ps ? 1024 : 256, ps ? 128 : 256, &p.psplits, &p.plen);
    }
    p.direct = p.splits == 1 && p.psplits == 0;
    return p;
}

size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

template <int D, bool BF, int P, int O>
hipError_t launch(const AttnArgs& a, Plan p, hipStream_t st) {
    const long long pgrid = static_cast<long long>(a.cache.heads) * p.psplits * p.pblocks;
    const int places = O <= S2 || O == S0 ? p.splits | 1 : p.splits;
    const long long grid = pgrid + static_cast<long long>(a.cache.heads) * places * p.blocks * a.batch.num_seqs;
    p.pgrid = static_cast<int>(pgrid);
    constexpr int bytes = lds_bytes(D, P) > lds_bytes(D, O) ? lds_bytes(D, P) : lds_bytes(D, O);
    if (bytes > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_kernel<D, BF, P, O>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    return launch_all(grid, [&](unsigned first, unsigned count) {
        p.first = first;
        hipLaunchKernelGGL((attn_kernel<D, BF, P, O>), dim3(count), dim3(256), bytes, st, a, p);
    });
}

// The prefix's unit has at least as many rows as a sequence's, so these
// combinations cover every call (a tiled prefix takes 128-row tiles, a streamed
// one of 17 to 32 rows streams the sequences' likewise).
template <int D, bool BF>
hipError_t run(const AttnArgs& a, Plan p, hipStream_t st) {
    const long long prows = static_cast<long long>(a.batch.tokens) * (a.q_heads / a.cache.heads);
    int own = kind_of(a.cache, a.batch, p.rows);
    if (own == S1 && a.batch.q_len == 1 && a.window == 0) own = S0;
    const int pre = p.psplits ? prows <= 16 ? S1 : prows <= stream_rows(D) ? S2 : T2 : NONE;
    hipError_t e;
    if constexpr (D > 128) {
        if (pre == NONE)
            e = own == S0   ? launch<D, BF, NONE, S0>(a, p, st)
                : own == S1 ? launch<D, BF, NONE, S1>(a, p, st)
                            : launch<D, BF, NONE, T1>(a, p, st);
        else
            e = pre == S1   ? launch<D, BF, S1, S1>(a, p, st)
                : own == S0 ? launch<D, BF, T1, S0>(a, p, st)
                : own == S1 ? launch<D, BF, T1, S1>(a, p, st)
                            : launch<D, BF, T1, T1>(a, p, st);
    } else if (pre == NONE) {
        e = own == S0   ? launch<D, BF, NONE, S0>(a, p, st)
            : own == S1 ? launch<D, BF, NONE, S1>(a, p, st)
            : own == S2 ? launch<D, BF, NONE, S2>(a, p, st)
            : own == T1 ? launch<D, BF, NONE, T1>(a, p, st)
                        : launch<D, BF, NONE, T2>(a, p, st);
    } else {
        e = pre == S1   ? launch<D, BF, S1, S1>(a, p, st)
            : pre == S2 ? launch<D, BF, S2, S2>(a, p, st)
            : own == S0 ? launch<D, BF, T2, S0>(a, p, st)
            : own == S1 ? launch<D, BF, T2, S1>(a, p, st)
            : own == S2 ? launch<D, BF, T2, S2>(a, p, st)
            : own == T1 ? launch<D, BF, T2, T1>(a, p, st)
                        : launch<D, BF, T2, T2>(a, p, st);
    }
    if (e != hipSuccess || p.direct) return e;
    const size_t rows = static_cast<size_t>(a.batch.tokens) * a.q_heads;
    if (p.psplits + p.splits <= kRowSplits && rows >= 4096) {
        constexpr size_t at = 1024 / D;
        return launch_all(static_cast<long long>((rows + at - 1) / at), [&](unsigned first, unsigned count) {
            p.first = first;
            hipLaunchKernelGGL((attn_join_rows_kernel<D>), dim3(count), dim3(256), 0, st, a, p);
        });
    }
    return launch_all(static_cast<long long>(rows), [&](unsigned first, unsigned count) {
        p.first = first;
        hipLaunchKernelGGL((attn_join_kernel<D>), dim3(count), dim3(256), 0, st, a, p);
    });
}

}  // namespace

bool attention_dim_ok(int dim) { return dim == 64 || dim == 128 || dim == 256; }

// Row and workgroup numbers are 32-bit.  A sequence has workgroups for q_len
// tokens whatever it holds, so many sequences beside one long prompt reach the
// second limit first (2^63 is out of reach: heads times blocks is at most the
// rows, as far as the first one holds).
bool attention_size_ok(const KvCache& c, const KvBatch& b, int q_heads) {
    constexpr long long most = 0x7fffffffll;
    if (static_cast<long long>(b.tokens) * q_heads > most) return false;
    const Plan p = make_plan(c, b, q_heads);
    const long long units = static_cast<long long>(c.heads) * p.blocks * b.num_seqs;
    return units <= most && units * (p.splits | 1) + static_cast<long long>(c.heads) * p.psplits * p.pblocks <= most;
}

size_t attention_workspace_bytes(const KvCache& c, const KvBatch& b, int q_heads) {
    const Plan p = make_plan(c, b, q_heads);
    if (p.direct) return 0;
    const size_t n = static_cast<size_t>(p.psplits + p.splits) * b.tokens * q_heads;
    return up256(n * c.dim * sizeof(float)) + up256(n * sizeof(float2));
}

hipError_t launch_attention(const AttnArgs& a, void* ws, hipStream_t st) {
    Plan p = make_plan(a.cache, a.batch, a.q_heads);
    if (!p.direct) {
        const size_t n = static_cast<size_t>(p.psplits + p.splits) * a.batch.tokens * a.q_heads;
        p.part = static_cast<float*>(ws);
        p.stat = reinterpret_cast<float2*>(static_cast<char*>(ws) + up256(n * a.cache.dim * sizeof(float)));
    }
    const bool bf = a.cache.dtype == DT_BF16;
    if (a.cache.dim == 64) return bf ? run<64, true>(a, p, st) : run<64, false>(a, p, st);
    if (a.cache.dim == 128) return bf ? run<128, true>(a, p, st) : run<128, false>(a, p, st);
    return bf ? run<256, true>(a, p, st) : run<256, false>(a, p, st);
}

}  // namespace cl
