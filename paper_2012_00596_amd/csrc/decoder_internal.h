// Kernel argument blocks and launchers of the decoder-block operators (norm with gate and residual, paged cache,
// attention of one token and of runs of tokens).
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

// The cache as the kernels see it; a row is head_dim elements.  Scales: of a cache of 8-bit floats, a byte for 32 elements.
struct CacheArgs {
    void *k, *v;
    const int32_t *table;
    int pages, page_size, kv_heads, head_dim, sequences, table_stride;
    uint8_t *k_scale, *v_scale;
};
constexpr uint32_t kAbsent = 0xffffffffu; // the row of a token that is not in the cache

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
    // runs of new tokens: rows [T][heads] of q and y, start [sequences + 1], workgroups a key head and cut
    const int32_t *start;
    int T, places;
};
constexpr int kMaxSplits = 512;
inline unsigned join_threads(int splits) { return splits <= 16 ? 64 : kMaxSplits; } // of a workgroup that joins a row's cuts

struct WriteArgs {
    CacheArgs c;
    const void *q, *k, *v;
    void *q_out;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *sequence, *position;
    const float *q_weight, *k_weight, *cos_sin;
    float eps, inv_d;
    int T, heads, positions, rot_dim, pairs;
};

struct ReadArgs {
    CacheArgs c;
    void *k_out, *v_out;
    const int32_t *sequence, *position;
    int T;
};

struct ChunkArgs {
    CacheArgs c;
    const void *q;
    void *y;
    float *lse;
    int64_t q_stride;
    const int32_t *start, *length;
    int T, heads, max_length, window;
    float scale;
    // cuts of `chunk` tokens; more than one: unnormalised sums [row][cut][head_dim] and (maximum, sum) of each, rows [T][heads]
    int chunk, splits, places; // places: workgroups a key head and cut
    float *part;
    float2 *part_stat;
};
constexpr int kChunkRows = 128; // (token, query head of a key head) of a workgroup's tile

// How a launch of single tokens cuts the tokens; `pairs`: workgroups a cut, `rows`: of y.
struct Cuts {
    int chunk, splits, waves;
    size_t stat_at, need, bytes; // (maximum, sum) pairs lie behind the sums; need: of this launch, bytes: enough for any window
};
Cuts plan_cuts(const CacheArgs &c, long pairs, size_t rows, int max_length, int window);

int launch_gated_residual_norm(int dt, const NormArgs &a, void *stream);
int launch_kv_append(int dt, const AppendArgs &a, void *stream);
int launch_paged_attention(int dt, const AttentionArgs &a, void *stream);
int launch_kv_write(int dt, const WriteArgs &a, void *stream);
int launch_kv_read(int dt, const ReadArgs &a, void *stream);
int launch_chunk_attention(int dt, const ChunkArgs &a, void *stream);
int launch_short_runs(int dt, const AttentionArgs &a, int groups, void *stream); // groups of 16 rows
int launch_chunk_join(int dt, const ChunkArgs &a, void *stream);

// Arguments that the calls on a cache share.  scales NULL: a cache of 16 bits; dt: storage type of the rows outside.
int check_cache(const npas_kv_cache *c, const npas_kv_scales *scales, int heads, CacheArgs *out, int *dt);
bool misaligned(const void *p, size_t to);
bool bad_stride(int64_t stride, int64_t row);

// Refuses what is more than a launch can have, 2^32 - 1 threads.
int check_grid(const char *what, uint64_t workgroups, unsigned threads);
// Reports the launch error that is pending, if any.
int launched(const char *what);

} // namespace npas
