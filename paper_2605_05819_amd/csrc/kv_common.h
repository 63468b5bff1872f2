// The paged cache and the batch of sequences as the kernels see them: which
// sequence a token belongs to, where its key stands, how many keys there are.
// Every value read from device memory is held inside the host's bounds before
// it becomes an address.
#pragma once

#include "cl_device.h"
#include "cl_internal.h"

namespace cl {

// A sequence's new tokens [start, start + count) and its keys, all clamped.
struct Seq {
    int start, count, keys;
};

__device__ __forceinline__ Seq load_seq(const KvBatch& b, int s) {
    Seq q;
    if (b.q_start) {
        q.start = min(max(b.q_start[s], 0), b.tokens);
        q.count = min(max(b.q_start[s + 1], q.start), b.tokens) - q.start;
    } else {
        q.start = s * b.q_len;
        q.count = b.q_len;
    }
    q.keys = min(max(b.kv_len[s], 0), b.key_limit);
    return q;
}

// The sequence whose range holds the token (the last with start <= token), or
// -1: one coalesced load and a ballot per 64 sequences in place of a search
// of dependent loads.  Called by whole waves with one token.
__device__ __forceinline__ int seq_of(const KvBatch& b, int token) {
    if (!b.q_start) return token / b.q_len;
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int base = 0; base < b.num_seqs; base += 64) {
        const int i = base + lane;
        n += __popcll(__ballot(i < b.num_seqs && b.q_start[i] <= token));
    }
    return n - 1;
}

}  // namespace cl
