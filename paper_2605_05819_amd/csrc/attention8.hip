// Attention over a cache of e4m3 codes with a power of two for each block of rows
// and head (the kernels: attention_kernels.h).
//
// A prompt's row blocks each convert all keys that they see.  Where there are many
// of them, the keys become a 16-bit cache in the workspace first, once, and the
// prompt is one over that cache: a launch that moves 3 bytes a value, in place of
// a tenth to a fifth of the tiles' time.  The values are the same.  Ragged prompts of up
// to 7001 tokens over 9001 keys 927 -> 855 us (862 from 16 bits, whose pages are
// scattered); four of 500 to 2000 tokens over up to 4000 keys, 64-wide heads 136 -> 120,
// 256-wide 441 -> 372.

#include "attention_kernels.h"

namespace cl {
namespace {

// The 16-bit cache of a call's own pages: the pages of sequence s are s * pages ...,
// in the order of their keys.
struct Ahead {
    int pages;                     // of a sequence (0: keys are converted as they are used)
    size_t pool;                   // bytes of K, and of V
};

// From 16 row blocks a sequence on, if a CU has one or more of them, up to 2 GiB and without
// a prefix.  (Two sequences of 300 tokens over 2000 keys, 10 blocks: 45.5 us
// as they are used, 48.8 ahead; 38 blocks of one head, 76 in all, 30.2 and 33.3;
// 16 blocks, 512 in all, 110 and 108.)
constexpr int kAheadBlocks = 16, kAheadUnits = 256;

Ahead ahead_of(const KvCache& c, const KvBatch& b, int q_heads) {
    Ahead h{};
    const Plan p = make_plan(c, b, q_heads);
    if (b.prefix_len > 0 || p.rows <= stream_rows(c.dim) || p.blocks < kAheadBlocks ||
        static_cast<long long>(b.num_seqs) * c.heads * p.blocks < kAheadUnits)
        return h;
    const int pages = (b.key_limit + (1 << c.page_shift) - 1) >> c.page_shift;
    const size_t row = static_cast<size_t>(c.heads) * c.dim * 2 << c.page_shift;       // bytes of a page
    if (pages < 1 || static_cast<size_t>(b.num_seqs) > (1ull << 30) / row / pages) return h;
    h.pages = pages;
    h.pool = up256(row * b.num_seqs * pages);
    return h;
}

// 16 KB of codes of K and of V of one sequence and head, 16 a lane: chunk x of
// sequence y, head z.
template <int D, bool BF>
__global__ __launch_bounds__(256) void convert_kernel(AttnArgs a, uint16_t* k16, uint16_t* v16, int32_t* table, int pages,
                                                      unsigned chunks) {
    constexpr int QC = D / 16, ROWS = 1024 / QC;      // pieces of a row; rows of a workgroup
    unsigned id = a.first + blockIdx.x;
    const int head = static_cast<int>(id % a.cache.heads);
    id /= a.cache.heads;
    const int chunk = static_cast<int>(id % chunks), s = static_cast<int>(id / chunks);
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
        const int page = s * pages + (key >> a.cache.page_shift), in = key & ((1 << a.cache.page_shift) - 1);
        const int r = pool_row(a, seg, head, key);
        if (head == 0 && in == 0 && c % QC == 0) table[page] = r >= 0 ? page : -1;
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
        *reinterpret_cast<u32x4*>(k16 + at) = decode8<BF>(k[i][0], k[i][1], fk);
        *reinterpret_cast<u32x4*>(k16 + at + 8) = decode8<BF>(k[i][2], k[i][3], fk);
        *reinterpret_cast<u32x4*>(v16 + at) = decode8<BF>(v[i][0], v[i][1], fv);
        *reinterpret_cast<u32x4*>(v16 + at + 8) = decode8<BF>(v[i][2], v[i][3], fv);
    }
}

template <int D>
hipError_t convert(AttnArgs a, uint16_t* k16, uint16_t* v16, int32_t* table, int pages, hipStream_t st) {
    constexpr int ROWS = 16384 / D;
    const unsigned chunks = static_cast<unsigned>(ceil_div(a.batch.key_limit, ROWS));
    return launch_all(static_cast<long long>(chunks) * a.batch.num_seqs * a.cache.heads, [&](unsigned first, unsigned count) {
        a.first = first;
        if (a.cache.dtype == DT_BF16)
            hipLaunchKernelGGL((convert_kernel<D, true>), dim3(count), dim3(256), 0, st, a, k16, v16, table, pages, chunks);
        else
            hipLaunchKernelGGL((convert_kernel<D, false>), dim3(count), dim3(256), 0, st, a, k16, v16, table, pages, chunks);
    });
}

}  // namespace

size_t attention8_workspace_bytes(const KvCache& c, const KvBatch& b, int q_heads) {
    const Ahead h = ahead_of(c, b, q_heads);
    return attention_workspace_bytes(c, b, q_heads) +
           (h.pages ? 2 * h.pool + up256(static_cast<size_t>(h.pages) * b.num_seqs * sizeof(int32_t)) : 0);
}

hipError_t launch_attention8(const AttnArgs& args, void* ws, hipStream_t st) {
    const Ahead h = ahead_of(args.cache, args.batch, args.q_heads);
    if (h.pages == 0) return launch_for<true>(args, ws, st);
    AttnArgs a = args;
    char* at = static_cast<char*>(ws) + attention_workspace_bytes(a.cache, a.batch, a.q_heads);
    uint16_t* const k16 = reinterpret_cast<uint16_t*>(at);
    uint16_t* const v16 = reinterpret_cast<uint16_t*>(at + h.pool);
    int32_t* const table = reinterpret_cast<int32_t*>(at + 2 * h.pool);
    const hipError_t e = a.cache.dim == 64    ? convert<64>(a, k16, v16, table, h.pages, st)
                         : a.cache.dim == 128 ? convert<128>(a, k16, v16, table, h.pages, st)
                                              : convert<256>(a, k16, v16, table, h.pages, st);
    if (e != hipSuccess) return e;
    a.cache.k = k16;
    a.cache.v = v16;
    a.cache.num_pages = a.batch.num_seqs * h.pages;
    a.batch.page_table = table;
    a.batch.table_width = h.pages;
    return launch_attention(a, ws, st);
}

}  // namespace cl
