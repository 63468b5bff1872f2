// The pages of a cache and who holds them: sequences that take over others'
// pages, rows that get and give back pages, a pool that is compacted, and copies
// of pages and rows.
//
// refs[p] counts the table entries that hold page p; 0 is free.  Every choice goes
// by number, the lowest free page to the first entry in row order, so the same
// calls give the same tables.  Counts change by integer atomics, whose order does
// not show; what depends on all of them (which pages are free now, which last page
// is a row's alone) is read by the next launch, one workgroup that scans rows and
// pages.  The copies, a third launch, move all buffers' pages (keys and values of
// every layer, scales) at once.
//
// Tables are small (64 rows of 64 pages: 16 KB): the first two launches are bound
// by their chains of reads, the copies by memory.

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {
namespace {

constexpr int kScan = 1024;                  // threads of the scanning workgroup

__device__ __forceinline__ bool in_pool(int page, int num_pages) {
    return static_cast<unsigned>(page) < static_cast<unsigned>(num_pages);
}

// A row's keys of its own, and the entries they use.
__device__ __forceinline__ int own_keys(const PageTable& t, int len) {
    return min(max(len - t.prefix_len, 0), static_cast<int>(min(static_cast<long long>(t.width) << t.page_shift, 0x7fffffffll)));
}
__device__ __forceinline__ int entries_of(const PageTable& t, long long keys) {
    return static_cast<int>((keys + (1 << t.page_shift) - 1) >> t.page_shift);
}

// Inclusive sum over the workgroup's threads (kScan of them), and the total.
__device__ __forceinline__ int scan_sum(int v, int* waves, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(v, off, 64);
        if (lane >= off) v += o;
    }
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kScan / 64; ++w) {
        const int x = waves[w];
        before += w < wave ? x : 0;
        all += x;
    }
    __syncthreads();
    *total = all;
    return v + before;
}

// ------------------------------------------------------------------- forking

// Workgroup i makes new row i and settles the counts of old row i: each of its
// c children holds the used pages in its place (c - 1 more holders); pages kept
// ahead of its keys go to the first child, or free.
__global__ __launch_bounds__(256) void fork_rows_kernel(ForkArgs a) {
    __shared__ int sums[3];
    const int i = blockIdx.x, tid = threadIdx.x;
    if (tid < 3) sums[tid] = 0;
    __syncthreads();
    const int p = i < a.to.rows ? a.parents[i] : -1;
    const bool valid = p >= 0 && p < a.from.rows;
    int earlier = 0, mine = 0, siblings = 0;       // children of p ahead of i, of row i, of p
    for (int j = tid; j < a.to.rows; j += 256) {
        const int q = a.parents[j];
        earlier += j < i && q == p;
        mine += q == i;
        siblings += q == p;
    }
    if (earlier) atomicAdd(&sums[0], earlier);
    if (mine) atomicAdd(&sums[1], mine);
    if (siblings) atomicAdd(&sums[2], siblings);
    __syncthreads();
    const bool first = sums[0] == 0;
    const int width = a.from.width;
    if (i < a.to.rows) {
        const int len = valid ? max(a.from.kv_len[p], 0) : 0;
        const int used = entries_of(a.from, own_keys(a.from, len));
        const int32_t* src = a.from.pages + static_cast<size_t>(valid ? p : 0) * width;
        int32_t* dst = a.to.pages + static_cast<size_t>(i) * width;
        for (int e = tid; e < width; e += 256) {
            const int page = valid && (e < used || first) ? src[e] : -1;
            dst[e] = in_pool(page, a.num_pages) ? page : -1;
        }
        if (tid == 0) {
            a.to.kv_len[i] = len;
            a.keep[i] = !valid ? -1 : first ? sums[2] : -1 - sums[2];
        }
    }
    if (i < a.from.rows) {
        const int used = entries_of(a.from, own_keys(a.from, a.from.kv_len[i]));
        const int32_t* src = a.from.pages + static_cast<size_t>(i) * width;
        const int held = sums[1] - 1, ahead = sums[1] > 0 ? 0 : -1;
        for (int e = tid; e < width; e += 256) {
            const int page = src[e], more = e < used ? held : ahead;
            if (more != 0 && in_pool(page, a.num_pages)) atomicAdd(a.refs + page, more);
        }
    }
}

// The same by one wave, for few small rows.
__device__ __forceinline__ void fork_row(const ForkArgs& a, int i) {
    const int lane = threadIdx.x & 63, width = a.from.width;
    const int p = i < a.to.rows ? a.parents[i] : -1;
    const bool valid = p >= 0 && p < a.from.rows;
    int earlier = 0, mine = 0, siblings = 0;
    for (int base = 0; base < a.to.rows; base += 64) {
        const int j = base + lane, q = j < a.to.rows ? a.parents[j] : -1;
        earlier += __popcll(__ballot(j < i && q == p));
        mine += __popcll(__ballot(j < a.to.rows && q == i));
        siblings += __popcll(__ballot(j < a.to.rows && q == p));
    }
    if (i < a.to.rows) {
        const int len = valid ? max(a.from.kv_len[p], 0) : 0;
        const int used = entries_of(a.from, own_keys(a.from, len));
        for (int e = lane; e < width; e += 64) {
            const int page = valid && (e < used || earlier == 0) ? a.from.pages[static_cast<size_t>(p) * width + e] : -1;
            a.to.pages[static_cast<size_t>(i) * width + e] = in_pool(page, a.num_pages) ? page : -1;
        }
        if (lane == 0) {
            a.to.kv_len[i] = len;
            a.keep[i] = !valid ? -1 : earlier == 0 ? siblings : -1 - siblings;
        }
    }
    if (i < a.from.rows) {
        const int used = entries_of(a.from, own_keys(a.from, a.from.kv_len[i]));
        for (int e = lane; e < width; e += 64) {
            const int page = a.from.pages[static_cast<size_t>(i) * width + e], more = e < used ? mine - 1 : mine > 0 ? 0 : -1;
            if (more != 0 && in_pool(page, a.num_pages)) atomicAdd(a.refs + page, more);
        }
    }
}

// ------------------------------------------------------------- giving pages

// One workgroup: rows that are to grow ask for a page of their own in place of a
// partly used last one that others hold too (a copy), then for the entries they lack; the
// lowest free pages go to them in row order.  A last page whose holders are all to
// grow stays with the first of them.  Where pages run out a row keeps the page that
// it holds, shared as it was: its keys are whole, and it can ask again.  What is free is
// scanned before any count changes here, so no page is both copied from and given
// away.  LANES work on a row: a wave where rows ask for many entries, one where they ask for a few (64
// rows of one entry 5.7 us, 12 by waves).
template <int LANES>
__device__ __forceinline__ void give_pages(const GiveArgs& a) {
    __shared__ int waves[kScan / 64], opens[kScan / 64];
    const int tid = threadIdx.x, lane = tid % LANES, team = tid / LANES;
    constexpr int TEAMS = kScan / LANES;
    // the lanes of a row that hold true, as bits from the row's first lane
    const auto votes = [&](bool v) { return LANES == 64 ? static_cast<uint64_t>(__ballot(v)) : static_cast<uint64_t>(v); };
    const PageTable& t = a.table;
    int over = 0;                                  // entries past the table's width, 2^10 a row at most (2^20 rows stay below 2^31)

    struct Ask {
        int used, need, page;                      // page: of the last entry in use, to be copied (-1: none)
        bool open;                                 // others than the parent's children hold it too, who may all be growing
    };
    const auto want_of = [&](int i, int len) {         // a new row without a parent stays empty
        if (a.want) return static_cast<long long>(a.want[i]);
        return a.keep[i] == -1 ? 0ll : static_cast<long long>(len) + a.room;
    };
    const auto ask_of = [&](int i) {
        const int len = max(t.kv_len[i], 0);
        const int own = own_keys(t, len);
        const long long want = want_of(i, len);
        Ask r;
        r.used = entries_of(t, own);
        r.need = r.used;
        r.page = -1;
        r.open = false;
        if (want > len) {
            const long long need = want > t.prefix_len ? (want - t.prefix_len + (1 << t.page_shift) - 1) >> t.page_shift : 0;
            r.need = static_cast<int>(min(max(need, static_cast<long long>(r.used)), static_cast<long long>(t.width)));
            if (lane == 0 && need > t.width) over += static_cast<int>(min(need - t.width, 1ll << 10));
            if (own & ((1 << t.page_shift) - 1)) {
                const int page = t.pages[static_cast<size_t>(i) * t.width + r.used - 1];
                const int keep = a.keep ? a.keep[i] : 1, kin = keep > 0 ? keep : -1 - keep;
                if (in_pool(page, a.num_pages)) {
                    r.open = a.refs[page] != kin;
                    if (r.open || keep < 0) r.page = page;
                }
            }
        }
        return r;
    };

    bool open = false;
    for (int i = team; i < t.rows; i += TEAMS) {
        const Ask r = ask_of(i);
        open |= r.open;
        int n = r.page >= 0 ? 1 : 0;
        for (int e = r.used; e < r.need; e += LANES)
            n += __popcll(votes(e + lane < r.need && !in_pool(t.pages[static_cast<size_t>(i) * t.width + e + lane], a.num_pages)));
        if (lane == 0) {
            a.count[i] = n;
            a.copy_from[i] = r.page;
            a.copy_to[i] = r.open ? r.page : -1;
        }
    }
    const bool wave_open = __ballot(open) != 0;
    if ((tid & 63) == 0) opens[tid >> 6] = wave_open;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int w = 0; w < kScan / 64; ++w) any |= opens[w];
    if (any) {
        // The holders that grow leave their pages; one that nobody holds then stays
        // with the first of them (by number, through a.free's place for the page), and
        // all counts are put back.  Other waves' values are read by atomics, past the L1.
        const auto pages = [&](auto what) {
            for (int i = tid; i < t.rows; i += kScan) {
                const int page = a.copy_to[i];
                if (page >= 0) what(i, page);
            }
            __threadfence();
            __syncthreads();
        };
        pages([&](int, int page) {
            atomicAdd(a.refs + page, -1);
            atomicExch(a.free + page, 0x7fffffff);
        });
        pages([&](int i, int page) {
            if (atomicAdd(a.refs + page, 0) == 0) atomicMin(a.free + page, i);
        });
        pages([&](int i, int page) {
            if (atomicAdd(a.free + page, 0) == i) {
                a.copy_from[i] = -1;
                --a.count[i];
            }
        });
        pages([&](int, int page) { atomicAdd(a.refs + page, 1); });
    }
    int asked = 0;
    for (int base = 0; base < t.rows; base += kScan) {
        const int n = base + tid < t.rows ? a.count[base + tid] : 0;
        int total;
        const int upto = scan_sum(n, waves, &total);
        if (base + tid < t.rows) a.count[base + tid] = asked + upto - n;      // where the row's pages begin
        asked += total;
    }
    // the lowest free pages, as many as are asked for
    int found = 0;
    for (int base = 0; base < a.num_pages && found < asked; base += 4 * kScan) {
        int free_[4], n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int p = base + 4 * tid + j;
            free_[j] = p < a.num_pages && a.refs[p] == 0;
            n += free_[j];
        }
        int total;
        int at = found + scan_sum(n, waves, &total) - n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (free_[j]) {
                if (at < asked) a.free[at] = base + 4 * tid + j;
                ++at;
            }
        found += total;
    }
    __syncthreads();
    const int have = min(found, asked);
    for (int i = team; i < t.rows; i += TEAMS) {
        int32_t* const row = t.pages + static_cast<size_t>(i) * t.width;
        const int old = a.copy_from[i];
        int at = a.count[i];
        // the same bounds as above, without the counts that change now
        const int len = max(t.kv_len[i], 0), own = own_keys(t, len), used = entries_of(t, own);
        const long long want = want_of(i, len);
        int need = used;
        if (want > len && want > t.prefix_len)
            need = static_cast<int>(min(max((want - t.prefix_len + (1 << t.page_shift) - 1) >> t.page_shift, static_cast<long long>(used)),
                                        static_cast<long long>(t.width)));
        int to = -1;
        if (old >= 0) {
            to = at < have ? a.free[at] : -1;
            ++at;
            if (lane == 0 && to >= 0) {
                row[used - 1] = to;
                atomicAdd(a.refs + old, -1);
                a.refs[to] = 1;
            }
        }
        if (lane == 0) a.copy_to[i] = to;
        for (int e = used; e < need; e += LANES) {
            const bool lacks = e + lane < need && !in_pool(row[e + lane], a.num_pages);
            const uint64_t who = votes(lacks);
            if (lacks) {
                const int k = at + __popcll(who & ((1ull << lane) - 1));
                const int page = k < have ? a.free[k] : -1;
                row[e + lane] = page;
                if (page >= 0) a.refs[page] = 1;
            }
            at += __popcll(who);
        }
    }
    if (a.missing) {
        if (over) atomicAdd(a.missing, over);
        if (tid == 0 && asked > have) atomicAdd(a.missing, asked - have);
    }
}

template <int LANES>
__global__ __launch_bounds__(kScan) void give_pages_kernel(GiveArgs a) {
    give_pages<LANES>(a);
}

// A small fork whole: its rows, then their pages.  The counts that the first part
// changes by atomics are read only in the second.
__global__ __launch_bounds__(kScan) void fork_and_give_kernel(ForkArgs f, GiveArgs a) {
    const int rows = max(f.from.rows, f.to.rows);
    for (int i = threadIdx.x / 64; i < rows; i += kScan / 64) fork_row(f, i);
    __threadfence();
    __syncthreads();
    give_pages<1>(a);
}

// ------------------------------------------------------------------ freeing

// A workgroup a row.  An entry is given back by whoever swaps it out, so a row
// that is named twice gives its pages back once.
__global__ __launch_bounds__(256) void free_rows_kernel(FreeArgs a) {
    const int i = a.rows ? a.rows[blockIdx.x] : static_cast<int>(blockIdx.x);
    if (i < 0 || i >= a.table.rows) return;
    int32_t* const row = a.table.pages + static_cast<size_t>(i) * a.table.width;
    for (int e = threadIdx.x; e < a.table.width; e += 256) {
        const int page = atomicExch(row + e, -1);
        if (in_pool(page, a.num_pages)) atomicAdd(a.refs + page, -1);
    }
    if (threadIdx.x == 0) a.table.kv_len[i] = 0;
}

// --------------------------------------------------------------- compacting

// One workgroup: with L pages in use, the k-th used page from L on moves to the
// k-th free one below L.
__global__ __launch_bounds__(kScan) void plan_moves_kernel(CompactArgs a) {
    __shared__ int waves[kScan / 64];
    const int tid = threadIdx.x;
    int live = 0;
    for (int p = tid; p < a.num_pages; p += kScan) live += a.refs[p] > 0;
    int L;
    scan_sum(live, waves, &L);
    int holes = 0, movers = 0;
    for (int base = 0; base < a.num_pages; base += 4 * kScan) {
        int mark[4], n = 0;                         // holes count 1, movers 2^16 (4096 pages a pass at most)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int p = base + 4 * tid + j;
            const bool used = p < a.num_pages && a.refs[p] > 0;
            mark[j] = p >= a.num_pages ? 0 : p < L ? (used ? 0 : 1) : (used ? 1 << 16 : 0);
            n += mark[j];
        }
        int total;
        const int before = scan_sum(n, waves, &total) - n;
        int h = holes + (before & 0xffff), m = movers + (before >> 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int p = base + 4 * tid + j;
            if (mark[j] == 1) a.to[h++] = p;
            if (p >= L && p < a.num_pages) a.rank[p] = mark[j] ? m : -1;
            if (mark[j] > 1) a.from[m++] = p;
        }
        holes += total & 0xffff;
        movers += total >> 16;
    }
    __syncthreads();
    for (int k = tid; k < movers; k += kScan) {
        const int f = a.from[k], t = a.to[k];
        a.refs[t] = a.refs[f];
        a.refs[f] = 0;
    }
    if (tid == 0) a.head[0] = movers, a.head[1] = L;
}

// Table entries by their pages' new numbers, by workgroup `block` of `blocks`.
__device__ __forceinline__ void rename_pages(const CompactArgs& a, unsigned block, unsigned blocks) {
    const int L = a.head[1];
    for (int n = 0; n < a.tables; ++n) {
        int32_t* const table = a.table[n];
        for (long long i = static_cast<long long>(block) * 256 + threadIdx.x; i < a.size[n]; i += static_cast<long long>(blocks) * 256) {
            const int page = table[i];
            if (page < L || page >= a.num_pages) continue;
            const int k = a.rank[page];
            table[i] = k >= 0 ? a.to[k] : -1;
        }
    }
}

// ------------------------------------------------------------------- copying

constexpr int kChunk = 16384;                // bytes of a workgroup's turn

template <class T>
__device__ __forceinline__ void copy_chunk(const char* from, char* to, int bytes) {
    const T* const f = reinterpret_cast<const T*>(from);
    T* const t = reinterpret_cast<T*>(to);
    const int n = bytes / static_cast<int>(sizeof(T));
    int i = threadIdx.x;
    for (; i + 768 < n; i += 1024) {
        const T a = f[i], b = f[i + 256], c = f[i + 512], d = f[i + 768];
        t[i] = a, t[i + 256] = b, t[i + 512] = c, t[i + 768] = d;
    }
    for (; i < n; i += 256) t[i] = f[i];
}

// Row from[i] of every buffer's source to row to[i] of its destination (i where
// there is no such array), i < n.  A workgroup takes turns of 16 KB; rows out of
// range, and rows that go nowhere (-1), are passed over.
template <int N>
__device__ __forceinline__ void copy_rows(const CopyList<N>& a, unsigned block, unsigned blocks) {
    const int n = a.count ? min(*a.count, a.n) : a.n;
    const long long turns = static_cast<long long>(n) * a.buffers * a.chunks;
    for (long long turn = block; turn < turns; turn += blocks) {
        const int c = static_cast<int>(turn % a.chunks);
        const long long rest = turn / a.chunks;
        const int b = static_cast<int>(rest % a.buffers), i = static_cast<int>(rest / a.buffers);
        const CopyBuffer& buf = a.buffer[b];
        const long long at = static_cast<long long>(c) * kChunk;
        if (at >= buf.bytes) continue;
        const int f = a.from ? a.from[i] : i, t = a.to ? a.to[i] : i;
        if (!in_pool(f, a.from_rows) || !in_pool(t, a.to_rows) || (buf.src == buf.dst && f == t)) continue;
        const char* const src = buf.src + static_cast<size_t>(f) * buf.bytes + at;
        char* const dst = buf.dst + static_cast<size_t>(t) * buf.bytes + at;
        const int bytes = static_cast<int>(min(buf.bytes - at, static_cast<long long>(kChunk)));
        if (buf.align == 16) copy_chunk<u32x4>(src, dst, bytes);
        else if (buf.align == 4) copy_chunk<uint32_t>(src, dst, bytes);
        else copy_chunk<uint8_t>(src, dst, bytes);
    }
}

template <int N>
__global__ __launch_bounds__(256) void copy_rows_kernel(CopyList<N> a) {
    copy_rows(a, blockIdx.x, gridDim.x);
}

// A compaction's moves and new names, which need nothing of each other: `renaming`
// workgroups, the first ones, see to the tables.
template <int N>
__global__ __launch_bounds__(256) void move_pages_kernel(CopyList<N> c, CompactArgs a, unsigned renaming) {
    if (blockIdx.x < renaming) rename_pages(a, blockIdx.x, renaming);
    else copy_rows(c, blockIdx.x - renaming, gridDim.x - renaming);
}

size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

// Parts of a workspace.
struct Room {
    char* at;
    int32_t* ints(long long n) {
        int32_t* p = reinterpret_cast<int32_t*>(at);
        at += up256(static_cast<size_t>(n) * 4);
        return p;
    }
};

}  // namespace

// The buffers from number `first` on into a launch's arguments, as many as it takes;
// its workgroups.
template <int N>
static unsigned fill(CopyList<N>& a, const CopyBuffer* buffers, int first, int n) {
    a.buffers = n - first < N ? n - first : N;
    long long most = 1;
    for (int b = 0; b < a.buffers; ++b) {
        a.buffer[b] = buffers[first + b];
        CopyBuffer& buf = a.buffer[b];
        const uintptr_t bits = reinterpret_cast<uintptr_t>(buf.src) | reinterpret_cast<uintptr_t>(buf.dst) |
                               static_cast<uintptr_t>(buf.bytes);
        buf.align = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
        if (buf.bytes > most) most = buf.bytes;
    }
    a.chunks = static_cast<int>((most + kChunk - 1) / kChunk);
    const long long turns = static_cast<long long>(a.n) * a.buffers * a.chunks;
    return static_cast<unsigned>(turns < 8192 ? turns : 8192);
}

template <int N>
static hipError_t copy_in_turn(const CopyRows& rows, const CopyBuffer* buffers, int n, hipStream_t st) {
    CopyList<N> a;
    static_cast<CopyRows&>(a) = rows;
    for (int first = 0; first < n; first += N) {
        const unsigned grid = fill(a, buffers, first, n);
        hipLaunchKernelGGL(copy_rows_kernel<N>, dim3(grid), dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_copy_rows(const CopyRows& rows, const CopyBuffer* buffers, int n, hipStream_t st) {
    return n <= kFewCopyBuffers ? copy_in_turn<kFewCopyBuffers>(rows, buffers, n, st)
                                : copy_in_turn<kMaxCopyBuffers>(rows, buffers, n, st);
}

// Row lists and free pages of kv_fork and kv_reserve; lists of kv_compact.
size_t pages_workspace_bytes(int num_pages, int rows) {
    const size_t give = 4 * up256(static_cast<size_t>(rows) * 4) + up256(static_cast<size_t>(num_pages) * 4);
    const size_t compact = 256 + 3 * up256(static_cast<size_t>(num_pages) * 4);
    return give > compact ? give : compact;
}

namespace {

// f: a fork whose rows come first, in the same launch if each has a wave of its own
// (4 rows of 20 entries 13.2 us with their copies, 16.5 in two launches; 64 rows of 64
// would take 27 for 18).
hipError_t give(const Pool& pool, const PageTable& table, const int32_t* want, int room, const ForkArgs* f, Room ws,
                hipStream_t st) {
    const int32_t* const keep = f ? f->keep : nullptr;
    GiveArgs g{};
    g.table = table;
    g.refs = pool.refs;
    g.missing = pool.missing;
    g.num_pages = pool.num_pages;
    g.want = want;
    g.room = room;
    g.keep = keep;
    g.count = ws.ints(table.rows);
    g.copy_from = ws.ints(table.rows);
    g.copy_to = ws.ints(table.rows);
    g.free = ws.ints(pool.num_pages);
    const int rows = f && f->from.rows > table.rows ? f->from.rows : table.rows;
    const bool little = f && rows <= kScan / 64 && table.width <= 256 && room <= 4 << table.page_shift;
    if (little) {
        hipLaunchKernelGGL(fork_and_give_kernel, dim3(1), dim3(kScan), 0, st, *f, g);
    } else if (f) {
        hipLaunchKernelGGL(fork_rows_kernel, dim3(rows), dim3(256), 0, st, *f);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!little && f && room <= 4 << table.page_shift) hipLaunchKernelGGL(give_pages_kernel<1>, dim3(1), dim3(kScan), 0, st, g);
    else if (!little) hipLaunchKernelGGL(give_pages_kernel<64>, dim3(1), dim3(kScan), 0, st, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pool.num_buffers == 0) return e;
    CopyRows c{};
    c.from = g.copy_from;
    c.to = g.copy_to;
    c.n = table.rows;
    c.from_rows = c.to_rows = pool.num_pages;
    return launch_copy_rows(c, pool.buffers, pool.num_buffers, st);
}

}  // namespace

hipError_t launch_kv_fork(const Pool& pool, const PageTable& from, const int32_t* parents, const PageTable& to, int room,
                          void* ws, hipStream_t st) {
    Room r{static_cast<char*>(ws)};
    ForkArgs f{};
    f.from = from;
    f.to = to;
    f.parents = parents;
    f.refs = pool.refs;
    f.num_pages = pool.num_pages;
    f.keep = r.ints(to.rows);
    if (room > 0) return give(pool, to, nullptr, room, &f, r, st);
    hipLaunchKernelGGL(fork_rows_kernel, dim3(from.rows > to.rows ? from.rows : to.rows), dim3(256), 0, st, f);
    return hipGetLastError();
}

hipError_t launch_kv_reserve(const Pool& pool, const PageTable& table, const int32_t* want, void* ws, hipStream_t st) {
    return give(pool, table, want, 0, nullptr, Room{static_cast<char*>(ws)}, st);
}

hipError_t launch_kv_free(const Pool& pool, const PageTable& table, const int32_t* rows, int n, hipStream_t st) {
    FreeArgs a{table, pool.refs, rows, pool.num_pages};
    hipLaunchKernelGGL(free_rows_kernel, dim3(rows ? n : table.rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int N>
static hipError_t move(const Pool& pool, const CopyRows& rows, const CompactArgs& a, unsigned renaming, hipStream_t st) {
    CopyList<N> c;
    static_cast<CopyRows&>(c) = rows;
    const unsigned grid = (pool.num_buffers ? fill(c, pool.buffers, 0, pool.num_buffers) : 0) + renaming;
    if (grid == 0) return hipSuccess;
    hipLaunchKernelGGL(move_pages_kernel<N>, dim3(grid), dim3(256), 0, st, c, a, renaming);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pool.num_buffers <= N) return e;
    return launch_copy_rows(rows, pool.buffers + N, pool.num_buffers - N, st);
}

hipError_t launch_kv_compact(const Pool& pool, int tables, int32_t* const* table, const int64_t* size, void* ws, hipStream_t st) {
    Room r{static_cast<char*>(ws)};
    CompactArgs a{};
    a.refs = pool.refs;
    a.num_pages = pool.num_pages;
    a.head = r.ints(2);
    a.from = r.ints(pool.num_pages);
    a.to = r.ints(pool.num_pages);
    a.rank = r.ints(pool.num_pages);
    a.tables = tables;
    int64_t most = 1;
    for (int n = 0; n < tables; ++n) {
        a.table[n] = table[n];
        a.size[n] = size[n];
        if (size[n] > most) most = size[n];
    }
    hipLaunchKernelGGL(plan_moves_kernel, dim3(1), dim3(kScan), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    CopyRows c{};
    c.from = a.from;
    c.to = a.to;
    c.count = a.head;
    c.n = pool.num_pages;
    c.from_rows = c.to_rows = pool.num_pages;
    const int64_t blocks = tables ? (most + 255) / 256 : 0;
    const unsigned renaming = static_cast<unsigned>(blocks < 1024 ? blocks : 1024);
    if (pool.num_buffers <= kFewCopyBuffers) return move<kFewCopyBuffers>(pool, c, a, renaming, st);
    return move<kMaxCopyBuffers>(pool, c, a, renaming, st);
}

}  // namespace cl
