// Attention over the paged cache.
//
// Token i of a sequence with n keys and a new tokens stands at p = n - a + i
// and sees key j if j < n, j <= p (causal) and j > p - window (windowed):
//
//     o = sum_j e^{s_j - m} v_j / sum_j e^{s_j - m},  s_j = scale q . k_j,  m = max_j s_j
//
// A workgroup takes one token and head; its four waves take every fourth key
// with a running maximum and sum of their own and meet in LDS at the end.

#include "cl_device.h"
#include "cl_internal.h"
#include "kv_common.h"

namespace cl {
namespace {

__global__ __launch_bounds__(256) void attention_kernel(AttnArgs a) {
    __shared__ float part[4][2 + 256];
    const int t = blockIdx.x, head = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int D = a.cache.dim, dt = a.cache.dtype;
    const int s = seq_of(a.batch, t);
    if (s < 0) return;
    const Seq q = load_seq(a.batch, s);
    if (t >= q.start + q.count) return;
    const int p = q.keys - q.count + (t - q.start);
    const int hi = a.causal ? min(p + 1, q.keys) : q.keys;
    const int lo = a.window > 0 ? max(0, p - a.window + 1) : 0;
    const int kvh = head / (a.q_heads / a.cache.heads);
    float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int d = 64 * i + lane;
        qv[i] = d < D ? act_to_f32(a.q[t * a.q_stride + static_cast<long long>(head) * D + d], dt) * a.scale : 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int j = lo + wave; j < hi; j += 4) {
        const int mine = j - a.batch.prefix_len;
        const int at = mine < 0 ? j : mine;
        int page = mine < 0 ? a.batch.prefix_table[at >> a.cache.page_shift]
                            : a.batch.page_table[static_cast<size_t>(s) * a.batch.table_width + (at >> a.cache.page_shift)];
        const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(a.cache.num_pages);
        if (bad) page = 0;
        const size_t slot = ((static_cast<size_t>(page) * a.cache.heads + kvh) << a.cache.page_shift) +
                            (at & ((1 << a.cache.page_shift) - 1));
        const uint16_t* k = a.cache.k + slot * D;
        const uint16_t* v = a.cache.v + slot * D;
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (64 * i + lane < D) x += qv[i] * act_to_f32(k[64 * i + lane], dt);
        x = wave_sum(x);
        if (bad) x = NAN;
        const float mn = x > m ? x : m;
        const float c = expf(m - (mn == -INFINITY ? 0.f : mn));
        const float e = x == -INFINITY ? 0.f : expf(x - mn);
        m = mn;
        l = l * c + e;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (64 * i + lane < D) o[i] = o[i] * c + e * act_to_f32(v[64 * i + lane], dt);
    }
    if (lane == 0) part[wave][0] = m, part[wave][1] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][2 + 64 * i + lane] = o[i];
    __syncthreads();
    if (wave) return;
    float mm = -INFINITY;
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, part[w][0]);
    float ll = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < 4; ++w) {
        const float c = part[w][0] == -INFINITY && part[w][1] == 0.f ? 0.f : expf(part[w][0] - mm);
        ll += c * part[w][1];
        for (int i = 0; i < 4; ++i) r[i] += c * part[w][2 + 64 * i + lane];
    }
    const size_t row = static_cast<size_t>(t) * a.q_heads + head;
    for (int i = 0; i < 4; ++i)
        if (64 * i + lane < D) store_out(a.out, row * D + 64 * i + lane, ll != 0.f ? r[i] / ll : 0.f, a.out_dtype);
    if (a.lse && lane == 0) a.lse[row] = ll != 0.f ? mm + logf(ll) : -INFINITY;
}

}  // namespace

bool attention_dim_ok(int dim) { return dim == 64 || dim == 128 || dim == 256; }

size_t attention_workspace_bytes(const KvCache&, const KvBatch&, int) { return 0; }

hipError_t launch_attention(const AttnArgs& a, void*, hipStream_t st) {
    hipLaunchKernelGGL(attention_kernel, dim3(a.batch.tokens, a.q_heads), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace cl
