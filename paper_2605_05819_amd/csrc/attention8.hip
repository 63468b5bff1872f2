// Attention over a cache of e4m3 codes with a power of two for each block of rows
// and head (the kernels: attention_kernels.h).
//
// A prompt's row blocks each convert all keys that they see.  Where there are many
// of them, the keys become a 16-bit cache in the workspace first, once, and the
// prompt is one over that cache: a launch that moves 3 bytes a value, in place of
// a tenth to a fifth of the tiles' time.  The values are the same.  Ragged prompts of up
// to 7001 tokens over 9001 keys 927 -> 855 us (862 from 16 bits, whose pages are
// scattered); four of 500 to 2000 tokens over up to 4000 keys, 64-wide heads 136 -> 120,
// 256-wide 441 -> 372.  Each sequence is converted or not by its own new tokens: the keys
// of a token that is decoded beside a prompt are read once, as codes (a prompt of 1000
// tokens beside 15 single ones over 8192 keys 299 us, 408 with all keys converted; 63 over 4000 beside
// 4000 tokens 416, 732; 300 over 8192 beside 2000 1447, 1402 by the kernel of codes alone).

#include "attention_kernels.h"

namespace cl {
namespace {

// The 16-bit cache of a call's long sequences: those of the n-th have the pages n * pages
// ..., in the order of their keys.
struct Ahead {
    int rows;                      // a long sequence has that many rows (tokens x heads of a key head) or more
    int slots;                     // long sequences at most
    int pages;                     // of each (0: keys are converted as they are used)
    size_t pool;                   // bytes of K, and of V
    uint16_t *k, *v;
    int32_t *table;                // [slots][pages]
    int32_t *slot;                 // [num_seqs], written where a sequence is long
};

// From 16 row blocks of the longest sequence on, if a CU has one or more of all, up to 2 GiB and without
// a prefix.  (Two sequences of 300 tokens over 2000 keys, 10 blocks: 45.5 us
// as they are used, 48.8 ahead; 38 blocks of one head, 76 in all, 30.2 and 33.3;
// 16 blocks, 512 in all, 110 and 108.)  Beside such a one a sequence is long from half
// as many blocks on (15 prompts of 220 tokens, 7 blocks, beside one of 600: over 1000 keys 96 us as
// codes, 98 ahead, over 4000 keys 294 and 335).  The batch's new tokens
// bound how many can be long.
constexpr int kAheadBlocks = 16, kAheadUnits = 256;

Ahead ahead_of(const KvCache& c, const KvBatch& b, int q_heads) {
    Ahead h{};
    const Plan p = make_plan(c, b, q_heads);
    if (b.prefix_len > 0 || p.rows <= stream_rows(c.dim) || p.blocks < kAheadBlocks ||
        static_cast<long long>(b.num_seqs) * c.heads * p.blocks < kAheadUnits)
        return h;
    const int group = q_heads / c.heads;
    h.rows = (kAheadBlocks / 2 - 1) * tile_rows(c, b, p.rows) + 1;
    const int most = b.tokens / ceil_div(h.rows, group);       // q_len's own rows are more, so 1 or more
    h.slots = b.q_start && most < b.num_seqs ? most : b.num_seqs;
    const int pages = (b.key_limit + (1 << c.page_shift) - 1) >> c.page_shift;
    const size_t row = static_cast<size_t>(c.heads) * c.dim * 2 << c.page_shift;       // bytes of a page
    if (pages < 1 || static_cast<size_t>(h.slots) > (1ull << 30) / row / pages) return h;
    h.pages = pages;
    h.pool = up256(row * h.slots * pages);
    return h;
}

size_t ahead_bytes(const Ahead& h, int num_seqs) {
    return h.pages ? 2 * h.pool + up256(static_cast<size_t>(h.pages) * h.slots * sizeof(int32_t)) +
                         up256(static_cast<size_t>(num_seqs) * sizeof(int32_t))
                   : 0;
}

// Whether a sequence's keys are converted: a call's rows of it, against the host's bound.
__device__ __forceinline__ bool is_long(const AttnArgs& a, const Ahead& h, int count) {
    return min(count, a.batch.q_len) * (a.q_heads / a.cache.heads) >= h.rows;
}

// The slot's sequence, or -1: the long ones in their order, 64 a step.
__device__ __forceinline__ int long_seq(const AttnArgs& a, const Ahead& h, int slot) {
    if (!a.batch.q_start) return slot;
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < a.batch.num_seqs; base += 64) {
        const int s = base + lane;
        const bool is = s < a.batch.num_seqs && is_long(a, h, load_seq(a.batch, s).count);
        const uint64_t all = __ballot(is), mine = __ballot(is && __popcll(all & ((1ull << lane) - 1)) == slot);
        if (mine) return base + __ffsll(static_cast<unsigned long long>(mine)) - 1;
        slot -= __popcll(all);
    }
    return -1;
}

// 16 KB of codes of K and of V of one long sequence and head, 16 a lane.
template <int D, bool BF>
__global__ __launch_bounds__(256) void convert_kernel(AttnArgs a, Ahead h, unsigned chunks) {
    constexpr int QC = D / 16, ROWS = 1024 / QC;      // pieces of a row; rows of a workgroup
    unsigned id = a.first + blockIdx.x;
    const int head = static_cast<int>(id % a.cache.heads);
    id /= a.cache.heads;
    const int chunk = static_cast<int>(id % chunks), slot = static_cast<int>(id / chunks);
    const int s = long_seq(a, h, slot);
    if (s < 0) return;
    if (head == 0 && chunk == 0 && threadIdx.x == 0) h.slot[s] = slot;
    const Segment seg = own_segment(a, s);
    // keys ahead of every row's window are not read; a tile begins at a multiple of
    // 64, and a page's first key names it in the table
    const int whole = max(64, 1 << a.cache.page_shift);
    const int seen = a.window > 0 ? max(seg.keys - seg.seq.count - a.window + 1, 0) & -whole : 0;
    const int base = chunk * ROWS;
    if (base >= seg.keys || base + ROWS <= seen) return;
    u32x4 k[4], v[4];
    uint32_t ks[4], vs[4];
    int to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = threadIdx.x + 256 * i, key = base + c / QC;
        to[i] = -1;
        if (key >= seg.keys) continue;
        const int page = slot * h.pages + (key >> a.cache.page_shift), in = key & ((1 << a.cache.page_shift) - 1);
        const int r = pool_row(a, seg, head, key);
        if (head == 0 && in == 0 && c % QC == 0) h.table[page] = r >= 0 ? page : -1;
        if (r < 0) continue;
        to[i] = ((page * a.cache.heads + head) << a.cache.page_shift) + in;
        const size_t at = static_cast<size_t>(r) * D + 16 * (c % QC);
        k[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(a.cache.k) + at);
        v[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(a.cache.v) + at);
        ks[i] = scale_byte(a.cache.k_scale, a, r);
        vs[i] = scale_byte(a.cache.v_scale, a, r);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (to[i] < 0) continue;
        const size_t at = static_cast<size_t>(to[i]) * D + 16 * ((threadIdx.x + 256 * i) % QC);
        const float fk = scale_of(ks[i]), fv = scale_of(vs[i]);
        *reinterpret_cast<u32x4*>(h.k + at) = decode8<BF>(k[i][0], k[i][1], fk);
        *reinterpret_cast<u32x4*>(h.k + at + 8) = decode8<BF>(k[i][2], k[i][3], fk);
        *reinterpret_cast<u32x4*>(h.v + at) = decode8<BF>(v[i][0], v[i][1], fv);
        *reinterpret_cast<u32x4*>(h.v + at + 8) = decode8<BF>(v[i][2], v[i][3], fv);
    }
}

// Tiles over both: a long sequence's keys from its 16-bit cache, the others' as codes.
// Those of 64-wide heads go 64 rows at a time: the 128-row tile of codes would take a third
// workgroup's place on the CU (four prompts of 500 to 2000 tokens 157 us, 164 so).  128-wide heads keep
// their 128 rows, whose loads are further ahead of their use (63 single tokens over 4000
// keys beside a prompt of 4000 tokens 414 us, 552 by halves), and 9 registers in memory with them,
// which converted keys do not notice (ragged prompts 853 us with and without).
template <int D>
constexpr int kBlocks = D > 128 ? 1 : 2;               // 16-row blocks of a wave: 64 or 128 rows, as the plan has them from kAheadUnits on

template <int D, bool BF>
__global__ __launch_bounds__(256, 2) void attn_mixed_kernel(AttnArgs a, Plan pl, Ahead h) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    TilePlace place = tile_place<false>(a, pl, static_cast<int>(pl.first + blockIdx.x));
    Segment seg = own_segment(a, place.seq);
    if (is_long(a, h, seg.seq.count)) {
        seg.table = h.table + static_cast<size_t>(min(max(h.slot[place.seq], 0), h.slots - 1)) * h.pages;
        a.cache.k = h.k;
        a.cache.v = h.v;
        a.cache.num_pages = h.slots * h.pages;
        attn_tile<D, BF, false, kBlocks<D>, false>(a, pl, place, seg, lds);
        return;
    }
    constexpr int EACH = D > 64 ? kBlocks<D> : 1, PARTS = kBlocks<D> / EACH;
    const int first = place.block * PARTS;
#pragma unroll 1
    for (int n = 0; n < PARTS; ++n) {
        place.block = first + n;
        if (n) __syncthreads();                        // the last one's flags have been read
        attn_tile<D, BF, true, EACH, false>(a, pl, place, seg, lds);
    }
}

// The conversion, then the tiles: of sequences of one length by the 16-bit cache's kernels.
template <int D, bool BF>
hipError_t run_ahead(AttnArgs a, Ahead h, void* ws, hipStream_t st) {
    constexpr int ROWS = 16384 / D;
    const unsigned chunks = static_cast<unsigned>(ceil_div(a.batch.key_limit, ROWS));
    const hipError_t e = launch_all(static_cast<long long>(chunks) * h.slots * a.cache.heads, [&](unsigned first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL((convert_kernel<D, BF>), dim3(count), dim3(256), 0, st, a, h, chunks);
    });
    if (e != hipSuccess) return e;
    if (!a.batch.q_start) {
        a.cache.k = h.k;
        a.cache.v = h.v;
        a.cache.num_pages = h.slots * h.pages;
        a.batch.page_table = h.table;
        a.batch.table_width = h.pages;
        return launch_attention(a, ws, st);
    }
    Plan p = make_plan(a.cache, a.batch, a.q_heads);            // kAheadUnits and more take one split: no join
    static_assert(tile_lds(D) <= 65536, "within what a launch has without asking");
    return launch_all(static_cast<long long>(a.cache.heads) * p.blocks * a.batch.num_seqs, [&](unsigned first, unsigned count) {
        p.first = first;
        hipLaunchKernelGGL((attn_mixed_kernel<D, BF>), dim3(count), dim3(256), tile_lds(D), st, a, p, h);
    });
}

}  // namespace

size_t attention8_workspace_bytes(const KvCache& c, const KvBatch& b, int q_heads) {
    return attention_workspace_bytes(c, b, q_heads) + ahead_bytes(ahead_of(c, b, q_heads), b.num_seqs);
}

hipError_t launch_attention8(const AttnArgs& a, void* ws, hipStream_t st) {
    Ahead h = ahead_of(a.cache, a.batch, a.q_heads);
    if (h.pages == 0) return launch_for<true>(a, ws, st);
    char* at = static_cast<char*>(ws) + attention_workspace_bytes(a.cache, a.batch, a.q_heads);
    h.k = reinterpret_cast<uint16_t*>(at);
    h.v = reinterpret_cast<uint16_t*>(at + h.pool);
    h.table = reinterpret_cast<int32_t*>(at + 2 * h.pool);
    h.slot = reinterpret_cast<int32_t*>(at + 2 * h.pool + up256(static_cast<size_t>(h.pages) * h.slots * sizeof(int32_t)));
    const bool bf = a.cache.dtype == DT_BF16;
    if (a.cache.dim == 64) return bf ? run_ahead<64, true>(a, h, ws, st) : run_ahead<64, false>(a, h, ws, st);
    if (a.cache.dim == 128) return bf ? run_ahead<128, true>(a, h, ws, st) : run_ahead<128, false>(a, h, ws, st);
    return bf ? run_ahead<256, true>(a, h, ws, st) : run_ahead<256, false>(a, h, ws, st);
}

}  // namespace cl
