// Attention over a cache of 16-bit values (the kernels: attention_kernels.h), and
// the sizes of a call, which both kinds of cache share.

#include "attention_kernels.h"

namespace cl {

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

hipError_t launch_attention(const AttnArgs& a, void* ws, hipStream_t st) { return launch_for<false>(a, ws, st); }

}  // namespace cl
