// Host-side launchers shared between the ABI layer (api.hip) and the kernel
// translation units.  Arguments reaching these functions are already
// validated; each returns the hipError_t of its launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace cl {

struct QW {                    // packed backbone, validated
    const uint32_t* q;
    const uint16_t* s;
    const uint16_t* z;
    int d_out, d_in, bits, G;
};

struct LR {                    // compensation factors, validated (rank may be 0)
    const uint16_t* A;
    const uint16_t* B;
    int r_max, rank;
};

hipError_t launch_quantize_pack(const float* W, int d_out, int d_in, int bits, int G, uint32_t* q,
                                uint16_t* s, uint16_t* z, hipStream_t st);
hipError_t launch_dequantize(const QW& w, float* out, hipStream_t st);

// Decode of a window of n (1..8) linears sharing d_in, bits, group size and
// the activations x; arguments already validated.  glu: n = 2 linears of the
// same d_out (gate, up) and one output y[0] = SiLU(gate x) * (up x).
size_t decode_workspace_bytes(int n, const QW* w, const LR* c, int T);
bool decode_fits(const QW& w);   // d_in within the kernel's K-slice limit
hipError_t launch_linear_decode(int n, const QW* w, const LR* c, const void* x, int T, int act,
                                void* const* y, int out, void* ws, hipStream_t st, bool glu = false);

// Prefill: T = X A^T into the workspace, then the MFMA GEMM with the rank
// fold; d_in must be a multiple of 64.
size_t prefill_workspace_bytes(const QW& w, const LR& c, int M);
hipError_t launch_linear_prefill(const QW& w, const LR& c, const void* X, int M, int act, void* Y, int out,
                                 void* ws, hipStream_t st);

// Compensation factors from the SVD of W - deq(Q) (fp64 Gram matrix and
// tridiagonal eigensolver); synchronizes the stream once per check of the
// eigenvectors.  hipErrorNotReady: the residual is not finite (0 sweeps) or the
// vectors did not pass within the sweep limit.
bool comp_fits(int d_out, int d_in);
size_t comp_workspace_bytes(int d_out, int d_in, int r_max);
hipError_t launch_build_compensation(const float* W, const QW& w, int r_max, uint16_t* A, uint16_t* B, float* sigma,
                                     void* ws, hipStream_t st, int* sweeps_out);

// MoE decode over stacked experts (expert e's arrays at e times one expert's
// size) for a window of n <= 4 linears sharing the routing and activations;
// arguments already validated.
bool moe_fits(const QW& w, int E, int T, int k);
size_t moe_workspace_bytes(int n, const QW* w, const int* r_max, int E, int T, int k, int x_per_slot);
hipError_t launch_moe_decode(int n, const QW* w, const uint16_t* const* A, const uint16_t* const* B,
                             const int* r_max, const int32_t* const* ranks, const int32_t* const* slot_ranks,
                             int E, const void* x, const void* u, int x_per_slot,
                             const int32_t* ids, int T, int k, int act, void* const* y, int out, void* ws,
                             hipStream_t st);

// The current device's routing-error record (see moe.hip): waits for the
// stream, returns the record in *word (0: none) and clears it.
hipError_t moe_take_routing_error(hipStream_t st, unsigned long long* word);

// Launches of n < 2^31 workgroups of up to 1024 work items each.  HIP takes less
// than 2^32 work items along a dimension, so there is a launch for every 2^21
// workgroups: launch(first, count), `count` of them from number `first` on.
// (A second grid dimension instead costs every launch 0.15 us.)
template <class F>
hipError_t launch_all(long long n, F launch) {
    constexpr long long kMost = 1ll << 21;
    for (long long first = 0; first < n; first += kMost) {
        launch(static_cast<unsigned>(first), static_cast<unsigned>(n - first < kMost ? n - first : kMost));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Paged keys and values, validated: [num_pages][heads][page_size][dim] each,
// page_size = 1 << page_shift.
struct KvCache {
    uint16_t* k;
    uint16_t* v;
    int num_pages, page_shift, heads, dim, dtype;
};

// Sequences of a call, validated.  key_limit is the most keys a sequence may
// have: min(max_kv_len, prefix_len + table_width * page_size).
struct KvBatch {
    const int32_t* q_start;        // [num_seqs + 1], or null: q_len tokens each
    const int32_t* kv_len;         // [num_seqs]
    const int32_t* page_table;     // [num_seqs][table_width]
    const int32_t* prefix_table;
    int num_seqs, tokens, q_len, table_width, prefix_len, key_limit;
};

struct Rope {                  // inv_freq null: no rotation
    const float* inv_freq;
    int rot_dim, interleaved;
    float magnitude;
};

// Rotation of q into q_out and of k into the cache beside v (append.hip).
// Strides are in elements between tokens; q may be null.
struct AppendArgs {
    KvCache cache;
    KvBatch batch;
    Rope rope;
    const uint16_t *q, *k, *v, *q_norm, *k_norm;
    const int32_t* positions;
    uint16_t* q_out;
    long long q_stride, k_stride, v_stride;
    int q_heads;
    float eps;
    unsigned first;                // token of the launch's first workgroup
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st);
void rope_frequencies(int rot_dim, double base, int kind, double factor, double trained_len, double low, double high,
                      float* inv_freq, float* magnitude);      // host code

// Attention over the paged cache (attention.hip).
struct AttnArgs {
    KvCache cache;
    KvBatch batch;
    const uint16_t* q;
    long long q_stride;
    int q_heads, causal, window, out_dtype;
    float scale;
    void* out;
    float* lse;                    // may be null
};
bool attention_dim_ok(int dim);
bool attention_size_ok(const KvCache& c, const KvBatch& b, int q_heads);   // every number of the launch fits
size_t attention_workspace_bytes(const KvCache& c, const KvBatch& b, int q_heads);
hipError_t launch_attention(const AttnArgs& a, void* ws, hipStream_t st);

// Residual add, gate, combination of slots and norms of one row (norm.hip).
struct NormArgs {
    const void *y, *residual, *weight, *bias, *post_weight, *gate;
    const float* slot_weights;     // [T][slots], or null: y is [T][d]
    void *h, *out;                 // h may be null
    int T, d, slots, layer, gate_per_token;
    int y_dtype, h_dtype, out_dtype, w_dtype;
    float eps, alpha, beta;
};
hipError_t launch_residual_norm(const NormArgs& a, hipStream_t st);

// Routing of tokens to experts (route.hip).
constexpr int kMaxRouteTables = 4;
constexpr int kMaxRankLevels = 16;
struct RouteArgs {
    const void* logits;
    const float* bias;
    int32_t* ids;
    float* weights;
    const int32_t* expert_ranks[kMaxRouteTables];
    int32_t* slot_ranks[kMaxRouteTables];
    int levels[kMaxRankLevels];
    int tables, nlevels;
    int T, E, k, dtype, sigmoid, groups, top_groups, group_best, renormalize;
    float scale;
    unsigned first;                // the launch's first workgroup
};
hipError_t launch_moe_route(RouteArgs a, hipStream_t st);

// Rank allocation (host code, ranks.hip): salient-set size and salience
// ratio of one descending spectrum; ranks of one compensation window (cont,
// if not null, receives the continuous ranks before alignment); layer scores
// from layer-level sensitivities.  Arguments already validated.
constexpr int kMaxRankWin = 64;
constexpr int kMaxLayers = 4096;
int salient_count(const float* sigma, int n, double tau, double* phi);
void allocate_window_ranks(int n, const float* const* sigma, const int* len, const double* sens, double layer_score,
                           double r_std, const int* levels, int nlevels, int r_max, double tau, int* ranks,
                           double* cont);
void layer_sensitivity(int L, const double* D, int K, double* S);

}  // namespace cl
