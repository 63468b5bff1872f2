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
// The first new token of a block leads: its workgroups take the block's new rows, a
// wave for K or V of one head.  The rows come in one batch of loads and stay in
// registers as they came; the values are formed twice from them, for the maximum
// and for the codes (kept, they would double the registers).  Rows that stood in
// the block before keep its exponent as a lower bound, and are rescaled where it
// grows.  Values are computed in fp32 and rounded once, to the code.
//
// Bound by its chains (starts -> length -> page -> rows -> maximum -> codes) with 4
// workgroups a CU, and by memory for the queries: 8593 tokens of 32 + 8 + 8 heads of
// 128 with per-head norms, 194 MB, 52 us, 3.7 TB/s (130 registers and more leave three
// workgroups a CU: 79 us); 64 single tokens 4.7 us.  Reading rows back: 8676 tokens' of 8 heads,
// 53 MB, in 15.8 us.

#include <math.h>

#include <type_traits>

#include "append_common.h"
#include "append_units.h"
#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));

// The type is a template parameter here: a value that is widened and rounded by a
// type known at run time takes some ten instructions, three this way.
template <bool BF>
__device__ __forceinline__ Quad widen(Raw r) {
    if constexpr (BF)
        return Quad{{__builtin_bit_cast(float, r.a << 16), __builtin_bit_cast(float, r.a & 0xffff0000u),
                     __builtin_bit_cast(float, r.b << 16), __builtin_bit_cast(float, r.b & 0xffff0000u)}};
    const f16x2 a = __builtin_bit_cast(f16x2, r.a), b = __builtin_bit_cast(f16x2, r.b);
    return Quad{{static_cast<float>(a[0]), static_cast<float>(a[1]), static_cast<float>(b[0]), static_cast<float>(b[1])}};
}

template <bool BF>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), b16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}

template <bool BF>
__device__ __forceinline__ Raw narrow(const Quad& q) {
    return Raw{narrow2<BF>(q.v[0], q.v[1]), narrow2<BF>(q.v[2], q.v[3])};
}

// The exponents' range of a type, and the largest magnitude that is held: larger
// ones (behind a rotation or a norm) become it.
template <bool BF>
constexpr int kLow = BF ? -117 : -15;
template <bool BF>
constexpr int kHigh = BF ? 120 : 8;
template <bool BF>
constexpr float kMost = BF ? 0x1.ep127f : 61440.f;

__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, static_cast<uint32_t>(max(e, -126) + 127) << 23); }

// Four values to codes.  ODD: some of the block's are infinite, NaN or above what
// is held; an infinity or NaN is the code of NaN.
template <bool ODD>
__device__ __forceinline__ uint32_t encode4(const Quad& q, float inverse, float most) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = q.v[i] * inverse;
        if (ODD) x[i] = fabsf(q.v[i]) <= 3.4028234663852886e38f ? fminf(fmaxf(q.v[i], -most), most) * inverse : NAN;
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

// Sine and cosine of pair j at a position, times the magnitude; the angle as
// append.hip forms it, and what its rounding to fp32 leaves out to first order.
__device__ __forceinline__ float2 turn_of(const AppendArgs& a, int pos, int j) {
    const double turns = static_cast<double>(pos) * static_cast<double>(a.rope.inv_freq[j]) * 0.15915494309189533577;  // 1 / (2 pi)
    const double part = turns - rint(turns);
    const float near = static_cast<float>(part), rest = static_cast<float>(part - near) * 6.28318531f;
    float sn, cs;
    sincospif(2.0f * near, &sn, &cs);
    return float2{fmaf(-sn, rest, cs) * a.rope.magnitude, fmaf(cs, rest, sn) * a.rope.magnitude};
}

// A lane's four pairs turned: (u_i, v_i) in halves, or neighbours in u, then v.
__device__ __forceinline__ void turn(Quad& u, Quad& v, const float2 (&t)[4], bool half) {
    if (half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = u.v[i], q = v.v[i];
            u.v[i] = p * t[i].x - q * t[i].y;
            v.v[i] = p * t[i].y + q * t[i].x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            float p = u.v[i], q = u.v[i + 1];
            u.v[i] = p * t[i / 2].x - q * t[i / 2].y;
            u.v[i + 1] = p * t[i / 2].y + q * t[i / 2].x;
            p = v.v[i], q = v.v[i + 1];
            v.v[i] = p * t[2 + i / 2].x - q * t[2 + i / 2].y;
            v.v[i + 1] = p * t[2 + i / 2].y + q * t[2 + i / 2].x;
        }
    }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), off, 64)));
    return v;
}

// One over the root mean square of a head vector, held by LG lanes.
template <int LG>
__device__ __forceinline__ float inverse_rms(const Quad& u, const Quad& v, int dim, float eps) {
    float s2 = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s2 += u.v[i] * u.v[i] + v.v[i] * v.v[i];
#pragma unroll
    for (int off = LG / 2; off > 0; off >>= 1) s2 += __shfl_xor(s2, off, 64);
    return __builtin_amdgcn_rsqf(s2 * (1.0f / static_cast<float>(dim)) + eps);      // dim is a power of two
}

// The queries' part, a wave's: HP heads of a token for each group of lanes, their
// loads ahead of the chain that finds the token's position.  A turn is made by one
// lane and shared through `turns`, the wave's own: each lane making the four it
// needs takes a third of all instructions.
template <int LG, bool VEC, bool BF, int HP>
__device__ __forceinline__ void queries(const AppendArgs& a, float2* turns, int t, int part) {
    const int lane = threadIdx.x % LG, at = 8 * lane;             // D = 8 LG
    const int D = a.cache.dim;
    const bool rotary = a.rope.inv_freq && at < a.rope.rot_dim;
    const bool half = rotary && !a.rope.interleaved;
    const int lo = half ? 4 * lane : at, hi = half ? a.rope.rot_dim / 2 + 4 * lane : at + 4;
    constexpr int step = 64 / LG;
    const int first = part * HP * step + static_cast<int>(threadIdx.x & 63) / LG;
    Raw x[HP], y_[HP];
#pragma unroll
    for (int n = 0; n < HP; ++n) {
        const int h = first + n * step;
        if (h < a.q_heads) load8<VEC>(a.q + static_cast<long long>(t) * a.q_stride + static_cast<size_t>(h) * D, lo, hi, half, x[n], y_[n]);
    }
    const int s = seq_of(a.batch, t);
    if (s < 0) return;
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count) return;               // no sequence's row
    float2 sc[4];
    if (a.rope.inv_freq) {
        const int pos = a.positions ? a.positions[t] : q.keys - q.count + (t - q.start);
        for (int i = threadIdx.x & 63; i < a.rope.rot_dim / 2; i += 64) turns[i] = turn_of(a, pos, i);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (rotary) {
            const float4* const p = reinterpret_cast<const float4*>(turns + 4 * lane);
            const float4 one = p[0], two = p[1];
            sc[0] = float2{one.x, one.y}, sc[1] = float2{one.z, one.w};
            sc[2] = float2{two.x, two.y}, sc[3] = float2{two.z, two.w};
        }
    }
#pragma unroll
    for (int n = 0; n < HP; ++n) {
        const int h = first + n * step;
        if (h >= a.q_heads) return;                   // whole groups: nothing is exchanged between them
        Quad u = widen<BF>(x[n]), v = widen<BF>(y_[n]);
        if (a.q_norm) {
            const float r = inverse_rms<LG>(u, v, D, a.eps);
            Raw rx, ry;
            load8<VEC>(a.q_norm, lo, hi, half, rx, ry);
            const Quad wx = widen<BF>(rx), wy = widen<BF>(ry);
#pragma unroll
            for (int i = 0; i < 4; ++i) u.v[i] = u.v[i] * wx.v[i] * r, v.v[i] = v.v[i] * wy.v[i] * r;
        }
        if (rotary) turn(u, v, sc, half);
        store8<VEC, (HP > 1)>(a.q_out + (static_cast<size_t>(t) * a.q_heads + h) * D, lo, hi, half, narrow<BF>(u), narrow<BF>(v));
    }
}

// New rows of one head (of K or V, a wave's) into one block.
// The norm and the turn are in fp32: the few values that stand within its errors,
// 1e-7, of a code step's border get the neighbour's code (8 to 15 of 9 M values of
// 8676 tokens of 8 heads; 15 to 18 before the angle kept its rest and the product
// with the weight became exact).  A Newton step on the inverse root changed none of
// it, K's part in fp64 took 97 us where this takes 65.
// R > 0: the wave holds the rows, 64 / LG an iteration and R of them at most, as
// they came, from one batch of loads.  R = 0: any number, loaded for each pass.
// A wave without a head helps with the turns and reads nothing of k and v.
template <int LG, bool VEC, bool BF, int R>
__device__ __forceinline__ void block_rows(const AppendArgs& a, const float2* turns, int t, int pos, int rows, int before, int first,
                                           const KvUnit& unit, bool shared_turns) {
    constexpr int ROWS = 64 / LG, HOLD = R > 0 ? R : 1;
    const int lane = threadIdx.x % LG, at = 8 * lane, group = (threadIdx.x & 63) / LG;
    const int D = a.cache.dim;
    const bool is_v = unit.is_v;
    const bool turned = a.rope.inv_freq && at < a.rope.rot_dim && !is_v;
    const bool half = turned && !a.rope.interleaved;
    const int lo = half ? 4 * lane : at, hi = half ? a.rope.rot_dim / 2 + 4 * lane : at + 4;
    const int pairs = a.rope.rot_dim / 2;
    const uint16_t* const src = is_v ? a.v : a.k;
    const long long stride = is_v ? a.v_stride : a.k_stride;
    const int loaded = loaded_rows(unit, rows);
    const uint16_t* const w = is_v ? nullptr : a.k_norm;

    Raw x[HOLD], y[HOLD];
    const auto load = [&](int i, Raw& rx, Raw& ry) {              // the block's i-th new row
        rx = ry = Raw{0u, 0u};
        if (i < loaded) load8<VEC>(src + row_offset(unit, stride, D, t + i), lo, hi, half, rx, ry);
    };
#pragma unroll
    for (int n = 0; n < R; ++n)
        if (n * ROWS < rows) load(n * ROWS + group, x[n], y[n]);
    if (R > 0 && shared_turns) {                                  // of all heads of K, by the whole workgroup
        float2* const to = const_cast<float2*>(turns);
        for (int i = threadIdx.x; i < rows * pairs; i += 256) {
            const int row = i / pairs;
            to[i] = turn_of(a, a.positions ? a.positions[t + row] : pos + row, i - row * pairs);
        }
        __syncthreads();
    }
    if (!unit.live) return;

    Quad wx = {}, wy = {};
    if (w) {
        Raw rx, ry;
        load8<VEC>(w, lo, hi, half, rx, ry);
        wx = widen<BF>(rx), wy = widen<BF>(ry);
    }
    const auto values = [&](int n, bool held, Quad& u, Quad& v) {
        const int i = n * ROWS + group, slot = held ? n : 0;
        if (!held) load(i, x[0], y[0]);
        u = widen<BF>(x[slot]), v = widen<BF>(y[slot]);
        if (w) {
            const float r = inverse_rms<LG>(u, v, D, a.eps);
#pragma unroll
            for (int j = 0; j < 4; ++j) u.v[j] = u.v[j] * wx.v[j] * r, v.v[j] = v.v[j] * wy.v[j] * r;      // the first product is exact
        }
        if (turned) {
            float2 sc[4];
            if constexpr (R > 0) {
                const float4* const p = reinterpret_cast<const float4*>(turns + min(i, rows - 1) * pairs + 4 * lane);
                const float4 one = p[0], two = p[1];
                sc[0] = float2{one.x, one.y}, sc[1] = float2{one.z, one.w};
                sc[2] = float2{two.x, two.y}, sc[3] = float2{two.z, two.w};
            } else {
                const int p = a.positions ? (i < rows ? a.positions[t + i] : 0) : pos + i;
#pragma unroll
                for (int j = 0; j < 4; ++j) sc[j] = turn_of(a, p, 4 * lane + j);
            }
            turn(u, v, sc, half);
        }
    };

    uint8_t* const scale = (is_v ? a.cache.v_scale : a.cache.k_scale) + (static_cast<unsigned>(first) >> a.cache.block_shift);
    uint8_t* const codes = reinterpret_cast<uint8_t*>(is_v ? a.cache.v : a.cache.k) + static_cast<size_t>(first) * D;
    uint32_t top = 0;                                 // largest magnitude's bits: infinities and NaN stand above all
    const auto largest = [&](int n) {
        Quad u, v;
        values(n, R > 0, u, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            top = max(top, __builtin_bit_cast(uint32_t, u.v[j]) & 0x7fffffffu);
            top = max(top, __builtin_bit_cast(uint32_t, v.v[j]) & 0x7fffffffu);
        }
    };
    if constexpr (R > 0) {
#pragma unroll
        for (int n = 0; n < R; ++n)
            if (n * ROWS < rows) largest(n);
    } else {
        for (int n = 0; n * ROWS < rows; ++n) largest(n);
    }
    top = wave_max(top);
    constexpr uint32_t kEnd = 0x7f800000u;
    const bool odd = top > __builtin_bit_cast(uint32_t, kMost<BF>);
    if (top >= kEnd) {                                // the largest of the finite ones
        top = 0;
        const auto finite = [&](int n) {
            Quad u, v;
            values(n, false, u, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t p = __builtin_bit_cast(uint32_t, u.v[j]) & 0x7fffffffu;
                const uint32_t o = __builtin_bit_cast(uint32_t, v.v[j]) & 0x7fffffffu;
                top = max(top, max(p < kEnd ? p : 0u, o < kEnd ? o : 0u));
            }
        };
        for (int n = 0; n * ROWS < rows; ++n) finite(n);
        if (R > 0) load(group, x[0], y[0]);
        top = wave_max(top);
    }
    const uint32_t bits = top;
    constexpr int low = kLow<BF>, high = kHigh<BF>;
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
    // the values are formed again from what came: kept, they would take twice the
    // registers, and a second workgroup's place on the CU
#pragma unroll
    for (int n = 0; n < R; ++n) asm volatile("" : "+v"(x[n].a), "+v"(x[n].b), "+v"(y[n].a), "+v"(y[n].b));
    const auto store = [&](int n, auto how) {
        Quad u, v;
        values(n, R > 0, u, v);
        const int i = n * ROWS + group;
        if (i >= rows) return;
        uint8_t* const to = codes + static_cast<size_t>(i) * D;
        const uint32_t p = encode4<decltype(how)::value>(u, inverse, kMost<BF>);
        const uint32_t o = encode4<decltype(how)::value>(v, inverse, kMost<BF>);
        if (half) {
            *reinterpret_cast<uint32_t*>(to + lo) = p;
            *reinterpret_cast<uint32_t*>(to + hi) = o;
        } else {
            *reinterpret_cast<u32x2*>(to + lo) = u32x2{p, o};
        }
    };
    const auto store_all = [&](auto how) {
        if constexpr (R > 0) {
#pragma unroll
            for (int n = 0; n < R; ++n)
                if (n * ROWS < rows) store(n, how);
        } else {
            for (int n = 0; n * ROWS < rows; ++n) store(n, how);
        }
    };
    if (odd) store_all(std::true_type{});
    else store_all(std::false_type{});
}

// Workgroups of K and V stand ahead of the queries', being the longer ones (8593
// tokens 84 us, 111 behind them, 107 spread among them).  One of them looks at `span`
// tokens and takes the blocks whose first new token is among them, four heads of K
// or V, a wave each.
template <int LG, bool VEC, bool BF, int R, int HP>
__global__ __launch_bounds__(256, R <= 8 ? 4 : 2) void kv_append8_kernel(AppendArgs a, long long kv_blocks, int span) {
    extern __shared__ __attribute__((aligned(16))) float2 turns[];       // [rows][rot_dim / 2] (R > 0); queries: a row a wave
    const long long id = static_cast<long long>(a.first) + blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= kv_blocks) {
        constexpr int each = HP * 64 / LG;            // heads of a wave
        const int parts = (a.q_heads + each - 1) / each;
        const long long u = 4 * (id - kv_blocks) + wave;
        if (u < static_cast<long long>(a.batch.tokens) * parts)
            queries<LG, VEC, BF, HP>(a, turns + wave * (a.rope.rot_dim / 2), static_cast<int>(u / parts),
                                 static_cast<int>(u % parts));
        return;
    }
    const int Hk = a.cache.heads, block = 1 << a.cache.block_shift, fours = (2 * Hk + 3) / 4;
    const int unit0 = 4 * static_cast<int>(id % fours);
    const KvUnit unit = kv_unit(unit0 + wave, Hk);
    const bool shared_turns = a.rope.inv_freq && unit0 < Hk;
    const long long from = id / fours * span;
    const int to = static_cast<int>(min(from + span, static_cast<long long>(a.batch.tokens)));
    // everything here is the same for the whole workgroup
    for (int t = static_cast<int>(from); t < to;) {
        const int s = seq_of(a.batch, t);
        if (s < 0) {                                  // rows ahead of the first sequence
            t = max(t + 1, min(a.batch.q_start[0], to));
            continue;
        }
        const Seq q = load_seq(a.batch, s);
        if (t >= q.start + q.count) {
            ++t;
            continue;
        }
        const int mine = q.keys - q.count + (t - q.start) - a.batch.prefix_len;
        if (mine < 0) {
            t += min(-mine, q.start + q.count - t);
            continue;
        }
        const int before = mine & (block - 1);        // rows of the block that stand ahead of this one
        const int rows = min(block - before, q.start + q.count - t);
        const int page = a.batch.page_table[static_cast<size_t>(s) * a.batch.table_width + (mine >> a.cache.page_shift)];
        if ((before == 0 || t == q.start) && page >= 0 && page < a.cache.num_pages) {
            const int first = ((page * Hk + unit.head) << a.cache.page_shift) + (mine & ((1 << a.cache.page_shift) - 1));
            block_rows<LG, VEC, BF, R>(a, turns, t, mine + a.batch.prefix_len, rows, before, first, unit, shared_turns);
            if (R > 0 && shared_turns && t + rows < to) __syncthreads();      // before the turns are others
        }
        t += rows;
    }
}

template <int LG, bool VEC, bool BF, int R, int HP>
hipError_t launch(AppendArgs a, int span, hipStream_t st) {
    constexpr int each = HP * 64 / LG;
    const long long kv = (static_cast<long long>(a.batch.tokens) + span - 1) / span * ((2 * a.cache.heads + 3) / 4);
    const long long q = a.q ? (static_cast<long long>(a.batch.tokens) * ((a.q_heads + each - 1) / each) + 3) / 4 : 0;
    const int table = R == 0 || a.cache.block_shift < 2 ? 4 : 1 << a.cache.block_shift;
    const size_t lds = a.rope.inv_freq ? static_cast<size_t>(a.rope.rot_dim) * 4 * table : 0;
    return launch_all(kv + q, [&](unsigned first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL((kv_append8_kernel<LG, VEC, BF, R, HP>), dim3(count), dim3(256), lds, st, a, kv, span);
    });
}

// Blocks of up to 16 iterations' rows are held (32 KB of turns at most).  A
// workgroup looks at one token where tokens are few; otherwise at as many as a
// block, or half of what a sequence has on average, so that hardly any finds
// nothing to do, and a wave of the queries' part takes four heads a group.
template <int LG, bool VEC, bool BF>
hipError_t choose(const AppendArgs& a, hipStream_t st) {
    constexpr int ROWS = 64 / LG;
    const int block = 1 << a.cache.block_shift;
    int span = 1;
    const bool many = a.batch.tokens >= 512;
    if (many)
        while (2 * span <= block && 4ll * span * a.batch.num_seqs <= a.batch.tokens) span *= 2;
    const int iterations = (block + ROWS - 1) / ROWS;
    if (iterations <= 4) return many ? launch<LG, VEC, BF, 4, 4>(a, span, st) : launch<LG, VEC, BF, 4, 1>(a, span, st);
    if (iterations <= 8) return many ? launch<LG, VEC, BF, 8, 4>(a, span, st) : launch<LG, VEC, BF, 8, 1>(a, span, st);
    if (iterations <= 16) return many ? launch<LG, VEC, BF, 16, 4>(a, span, st) : launch<LG, VEC, BF, 16, 1>(a, span, st);
    return many ? launch<LG, VEC, BF, 0, 4>(a, span, st) : launch<LG, VEC, BF, 0, 1>(a, span, st);
}

template <bool BF>
hipError_t by_width(const AppendArgs& a, bool vec, hipStream_t st) {
    if (a.cache.dim <= 64) return vec ? choose<8, true, BF>(a, st) : choose<8, false, BF>(a, st);
    if (a.cache.dim <= 128) return vec ? choose<16, true, BF>(a, st) : choose<16, false, BF>(a, st);
    return vec ? choose<32, true, BF>(a, st) : choose<32, false, BF>(a, st);
}

bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// ------------------------------------------------------------- reading back

// A workgroup for TOKENS neighbours, 8 values a lane: their chains (starts -> length
// -> page -> values) run side by side.
template <bool CODES, int TOKENS>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
    const int P = a.batch.prefix_len, D = a.cache.dim, Hk = a.cache.heads;
    const long long t0 = static_cast<long long>(a.first + blockIdx.x) * TOKENS;
    int first[TOKENS];                                 // pool row of head 0; -1: outside, -2: before position 0, -3: no token
#pragma unroll
    for (int n = 0; n < TOKENS; ++n) {
        first[n] = -3;
        if (t0 + n >= a.batch.tokens) continue;
        const int t = static_cast<int>(t0 + n), s = seq_of(a.batch, t);
        if (s < 0) continue;
        const Seq q = load_seq(a.batch, s);
        if (t >= q.start + q.count) continue;
        const int pos = q.keys - q.count + (t - q.start);
        first[n] = -2;
        if (pos < 0) continue;
        const int32_t* table = pos < P ? a.batch.prefix_table : a.batch.page_table + static_cast<size_t>(s) * a.batch.table_width;
        const int i = pos < P ? pos : pos - P, page = table[i >> a.cache.page_shift];
        first[n] = page >= 0 && page < a.cache.num_pages
                       ? (page * Hk << a.cache.page_shift) + (i & ((1 << a.cache.page_shift) - 1)) : -1;
    }
    const int each = Hk * D / 8;
    for (int i = threadIdx.x; i < 2 * each; i += 256) {
        const bool is_v = i >= each;
        const int at = 8 * (is_v ? i - each : i), head = at / D;
        u32x4 x[TOKENS];
        u32x2 c[TOKENS];
        uint32_t scale[TOKENS];
#pragma unroll
        for (int n = 0; n < TOKENS; ++n) {
            const int r = max(first[n], 0) + (head << a.cache.page_shift);
            const size_t from = static_cast<size_t>(r) * D + at % D;
            if constexpr (CODES) {
                c[n] = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(is_v ? a.cache.v : a.cache.k) + from);
                scale[n] = (is_v ? a.cache.v_scale : a.cache.k_scale)[static_cast<unsigned>(r) >> a.cache.block_shift];
            } else {
                x[n] = *reinterpret_cast<const u32x4*>((is_v ? a.cache.v : a.cache.k) + from);
            }
        }
#pragma unroll
        for (int n = 0; n < TOKENS; ++n) {
            if (first[n] == -3) continue;
            if constexpr (CODES) {
                const float f = __builtin_bit_cast(float, scale[n] << 23);
                const f32x2 v[4] = {__builtin_amdgcn_cvt_pk_f32_fp8(c[n][0], false), __builtin_amdgcn_cvt_pk_f32_fp8(c[n][0], true),
                                    __builtin_amdgcn_cvt_pk_f32_fp8(c[n][1], false), __builtin_amdgcn_cvt_pk_f32_fp8(c[n][1], true)};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[n][j] = a.cache.dtype == DT_BF16 ? narrow2<true>(v[j][0] * f, v[j][1] * f) : narrow2<false>(v[j][0] * f, v[j][1] * f);
            }
            if (first[n] < 0) {
                const uint32_t fill = first[n] == -2 ? 0u : 0xffffffffu;         // NaN in fp16 and bf16
                x[n] = u32x4{fill, fill, fill, fill};
            }
            *reinterpret_cast<u32x4*>((is_v ? a.v : a.k) + static_cast<size_t>(t0 + n) * Hk * D + at) = x[n];
        }
    }
}

}  // namespace

hipError_t launch_kv_append8(const AppendArgs& a, hipStream_t st) {
    const bool vec = wide(a.q) && wide(a.k) && wide(a.v) && wide(a.q_out) && wide(a.q_norm) && wide(a.k_norm) &&
                     a.q_stride % 8 == 0 && a.k_stride % 8 == 0 && a.v_stride % 8 == 0;
    return a.cache.dtype == DT_BF16 ? by_width<true>(a, vec, st) : by_width<false>(a, vec, st);
}

hipError_t launch_kv_read(const ReadArgs& args, bool codes, hipStream_t st) {
    ReadArgs a = args;
    const bool many = a.batch.tokens >= 2048;          // four tokens a workgroup (8676 tokens 16.7 -> 15.8 us)
    return launch_all((a.batch.tokens + (many ? 3ll : 0ll)) / (many ? 4 : 1), [&](unsigned first, unsigned count) {
        a.first = first;
        const dim3 grid(count), block(256);
        if (codes && many) hipLaunchKernelGGL((kv_read_kernel<true, 4>), grid, block, 0, st, a);
        else if (codes) hipLaunchKernelGGL((kv_read_kernel<true, 1>), grid, block, 0, st, a);
        else if (many) hipLaunchKernelGGL((kv_read_kernel<false, 4>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((kv_read_kernel<false, 1>), grid, block, 0, st, a);
    });
}

}  // namespace cl
