// Kernel argument blocks and launchers of the decoder-block operators (norm with gate and residual, paged cache,
// attention of one token).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "npas_internal.h"

namespace npas {

struct NormArgs {
    const void *branch, *h, *gate;
    const float *post, *pre;
    void *h_out, *n_out;
    int64_t gate_stride;
    float scale, eps, inv_d;
    int T, D;
};

// The cache as the kernels see it; a row is head_dim elements.
struct CacheArgs {
    void *k, *v;
    const int32_t *table;
    int pages, page_size, kv_heads, head_dim, sequences, table_stride;
};

struct AppendArgs {
    CacheArgs c;
    const void *q, *k, *v;
    void *q_out;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *sequence, *position;
    const float *cos_sin;
    int T, heads, positions, rot_dim, pairs;
};

struct AttentionArgs {
    CacheArgs c;
    const void *q;
    void *y;
    float *lse;
    int64_t q_stride;
    const int32_t *length;
    int heads, max_length, window;
    float scale;
    // cuts of `chunk` tokens; more than one: unnormalised sums [sequence][head][cut][head_dim] and (maximum, sum) of each
    int chunk, splits, waves; // waves of a workgroup, 4 or 8
    float *part;
    float2 *part_stat;
};
constexpr int kMaxSplits = 512;

int launch_gated_residual_norm(int dt, const NormArgs &a, void *stream);
int launch_kv_append(int dt, const AppendArgs &a, void *stream);
int launch_paged_attention(int dt, const AttentionArgs &a, void *stream);

// Refuses what is more than a launch can have, 2^32 - 1 threads.
int check_grid(const char *what, uint64_t workgroups, unsigned threads);
// Reports the launch error that is pending, if any.
int launched(const char *what);

} // namespace npas
