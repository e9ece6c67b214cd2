// C-ABI calls on the paged cache beside those of a decode step: argument checks, plans and launches of the write with norms, the read of 8-bit
// floats and the attention of runs of tokens.
#include <cmath>

#include "decoder_internal.h"

using namespace npas;

namespace {

// How a launch takes the rows and cuts the tokens.  Rows: (token, query head) of a key head.
//   - Runs of up to 32 rows on average (of heads longer than 128: 16, and up to 32 in tiles of 16, which is all that the registers hold): the kernel of single
//     tokens with one or two groups of 16 rows, cut as that is.  32 sequences of 5 tokens on 4000, 4 query heads a key head, head_dim 128, in 8 bits 71 us,
//     in tiles of kChunkRows 126; 16 of 8 40 and 61, in 16 bits 54 and 67; 5 tokens of one sequence 9.5 and 12.6; 4 of each of 32 at head_dim 256 251 and 325.
//     (7 tokens of one sequence on 8000 19.4 and 18.5.)
//   - Longer ones: tiles of kChunkRows.  Where they do not fill the card, a tile's tokens are cut for kWorkgroups in all, two a compute unit (256 tokens on 30000,
//     4 key heads and 8 query heads each: 236 us; for 1024 245, for 256 245).
//   - A cut more costs each row head_dim floats written and read, a token more in a cut its walk: their sum is least at a length that goes with the root of
//     rows and tokens (64 tokens of 32 heads on 8192: 16 cuts of 512 35 us, half as long 37, twice 40; on 30000, 8 heads, 512 32, 256 each 34, 1024 38), and
//     kLeast at the least (on 1000: 256 each 20 us, 512 26).
// The mean decides for all runs of a call: one of 500 tokens beside 63 single tokens on 4096 takes 347 us in 16 bits and 344 in 8, in two calls 79 + 189 and 76 + 112.
struct ChunkPlan {
    int groups; // of 16 rows; 0: tiles of kChunkRows
    long places;
    Cuts cuts;
};
ChunkPlan plan_chunks(const CacheArgs &c, int T, int heads, int max_length, int window)
{
    constexpr long kWorkgroups = 512, kLeast = 256, kMost = 256;
    const long room = (long)c.table_stride * c.page_size, longest = max_length < room ? max_length : room;
    const long group = heads / c.kv_heads, rows = (long)T * group, mean = (rows + c.sequences - 1) / c.sequences;
    ChunkPlan k{};
    k.groups = mean <= 16 || (mean <= 32 && c.head_dim > 128) ? 1 : mean <= 32 ? 2 : 0;
    const long tile = k.groups ? 16 * k.groups : kChunkRows, tiles = c.sequences * ((mean + tile - 1) / tile);
    k.places = rows / tile + c.sequences;
    const long seen = window > 0 && window < longest - tile ? window + tile : longest; // tokens that a tile's rows see
    if (k.groups) {
        k.cuts = plan_cuts(c, tiles * c.kv_heads, (size_t)T * heads, max_length, (int)seen);
        if (k.groups == 2) k.cuts.waves = 4;
        return k;
    }
    long want = (kWorkgroups + tiles * c.kv_heads - 1) / (tiles * c.kv_heads); // cuts
    if (want > kMost) want = kMost;
    long chunk = (seen + want - 1) / want, most = (longest + kLeast - 1) / kLeast;
    const long paid = (long)std::sqrt((double)seen * T * heads * 0.01);
    if (chunk < paid) chunk = paid;
    if (chunk < kLeast) chunk = kLeast;
    chunk = (chunk + 127) / 128 * 128;
    if (most > want) most = want; // over all windows
    constexpr long kEnd = 0x7fffff80; // (2^31 - 1 tokens in one cut would be rounded past it)
    if (chunk > kEnd) chunk = kEnd;
    if (longest > kEnd && most < 2) most = 2;
    k.cuts.chunk = (int)chunk;
    k.cuts.splits = (int)((seen + chunk - 1) / chunk);
    const size_t all = (size_t)T * heads, each = (size_t)c.head_dim * 4 + 8;
    k.cuts.stat_at = all * k.cuts.splits * c.head_dim * 4;
    if (k.cuts.splits > 1) k.cuts.need = all * k.cuts.splits * each;
    if (most > 1) k.cuts.bytes = all * most * each;
    return k;
}

int check_chunk(const CacheArgs &c, int T, int heads, int max_length)
{
    if (T > 0 && max_length > 0 && (double)T * heads <= 2147483647.0) return NPAS_OK;
    set_error("bad shape T=%d heads=%d max_length=%d (%d sequences)", T, heads, max_length, c.sequences);
    return NPAS_E_SHAPE;
}

} // namespace

extern "C" {

int npas_kv_write(const npas_kv_cache *cache, const npas_kv_scales *scales, const void *q_dev, int64_t q_stride, const void *k_dev,
                  int64_t k_stride, const void *v_dev, int64_t v_stride, void *q_out_dev, int T, int heads, const int32_t *sequence_dev,
                  const int32_t *position_dev, const float *q_weight_dev, const float *k_weight_dev, float eps, const float *cos_sin_dev,
                  int positions, int rot_dim, npas_rotation kind, void *hip_stream)
{
    WriteArgs a{};
    int dt;
    if (int rc = check_cache(cache, scales, heads, &a.c, &dt)) return rc;
    if (!k_dev || !v_dev || !position_dev || !q_dev != !q_out_dev || (q_weight_dev && !q_dev) || (rot_dim > 0 && !cos_sin_dev)) {
        set_error("NULL argument (q=%p q_out=%p q_weight=%p k=%p v=%p position=%p cos_sin=%p)", q_dev, q_out_dev, (const void *)q_weight_dev,
                  k_dev, v_dev, (const void *)position_dev, (const void *)cos_sin_dev);
        return NPAS_E_NULL;
    }
    const int64_t qrow = (int64_t)heads * a.c.head_dim, krow = (int64_t)a.c.kv_heads * a.c.head_dim;
    if (T <= 0 || rot_dim < 0 || rot_dim % 2 || rot_dim > a.c.head_dim || (rot_dim > 0 && positions <= 0) || !(eps >= 0.f) ||
        (q_dev && bad_stride(q_stride, qrow)) || bad_stride(k_stride, krow) || bad_stride(v_stride, krow) ||
        (kind != NPAS_ROTATE_HALVES && kind != NPAS_ROTATE_PAIRS)) {
        set_error("bad shape T=%d heads=%d rot_dim=%d positions=%d eps=%g strides %lld %lld %lld rotation %d", T, heads, rot_dim, positions,
                  (double)eps, (long long)q_stride, (long long)k_stride, (long long)v_stride, (int)kind);
        return NPAS_E_SHAPE;
    }
    if (misaligned(q_dev, 2) || misaligned(k_dev, 2) || misaligned(v_dev, 2) || misaligned(q_out_dev, 2) || misaligned(sequence_dev, 4) ||
        misaligned(position_dev, 4) || misaligned(cos_sin_dev, 4) || misaligned(q_weight_dev, 4) || misaligned(k_weight_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    a.q = q_dev; a.k = k_dev; a.v = v_dev; a.q_out = q_out_dev;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.sequence = sequence_dev; a.position = position_dev;
    a.q_weight = q_weight_dev; a.k_weight = k_weight_dev; a.cos_sin = cos_sin_dev; a.eps = eps; a.inv_d = (float)(1.0 / a.c.head_dim);
    a.T = T; a.heads = heads; a.positions = positions; a.rot_dim = rot_dim; a.pairs = kind == NPAS_ROTATE_PAIRS;
    return launch_kv_write(dt, a, hip_stream);
}

int npas_kv_read(const npas_kv_cache *cache, const npas_kv_scales *scales, void *k_out_dev, void *v_out_dev, int T,
                 const int32_t *sequence_dev, const int32_t *position_dev, void *hip_stream)
{
    ReadArgs a{};
    int dt;
    if (!scales || (!k_out_dev && !v_out_dev) || !position_dev) {
        set_error("NULL argument (scales=%p k_out=%p v_out=%p position=%p)", (const void *)scales, k_out_dev, v_out_dev, (const void *)position_dev);
        return NPAS_E_NULL;
    }
    if (int rc = check_cache(cache, scales, cache ? cache->kv_heads : 0, &a.c, &dt)) return rc;
    if (T <= 0) {
        set_error("bad shape T=%d", T);
        return NPAS_E_SHAPE;
    }
    if (misaligned(k_out_dev, 2) || misaligned(v_out_dev, 2) || misaligned(sequence_dev, 4) || misaligned(position_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    a.k_out = k_out_dev; a.v_out = v_out_dev; a.sequence = sequence_dev; a.position = position_dev; a.T = T;
    return launch_kv_read(dt, a, hip_stream);
}

size_t npas_chunk_attention_workspace_bytes(const npas_kv_cache *cache, const npas_kv_scales *scales, int T, int heads, int max_length)
{
    CacheArgs c;
    int dt;
    if (check_cache(cache, scales, heads, &c, &dt) || check_chunk(c, T, heads, max_length)) return 0;
    return plan_chunks(c, T, heads, max_length, 0).cuts.bytes;
}

int npas_chunk_attention(const npas_kv_cache *cache, const npas_kv_scales *scales, const void *q_dev, int64_t q_stride, void *y_dev,
                         float *lse_dev, int T, int heads, const int32_t *start_dev, const int32_t *length_dev, int max_length, int window,
                         float scale, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    ChunkArgs a{};
    int dt;
    if (int rc = check_cache(cache, scales, heads, &a.c, &dt)) return rc;
    if (!q_dev || !y_dev || !start_dev || !length_dev) {
        set_error("NULL argument (q=%p y=%p start=%p length=%p)", q_dev, y_dev, (const void *)start_dev, (const void *)length_dev);
        return NPAS_E_NULL;
    }
    if (int rc = check_chunk(a.c, T, heads, max_length)) return rc;
    if (window < 0 || bad_stride(q_stride, (int64_t)heads * a.c.head_dim) || !(scale == scale)) {
        set_error("bad shape heads=%d window=%d q_stride=%lld scale=%g", heads, window, (long long)q_stride, (double)scale);
        return NPAS_E_SHAPE;
    }
    if (misaligned(q_dev, 2) || misaligned(y_dev, 2) || misaligned(lse_dev, 4) || misaligned(start_dev, 4) || misaligned(length_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    const ChunkPlan plan = plan_chunks(a.c, T, heads, max_length, window);
    const Cuts &cuts = plan.cuts;
    if (cuts.need && (!workspace_dev || workspace_bytes < cuts.need || misaligned(workspace_dev, 16))) {
        set_error("chunk attention needs %zu bytes of workspace at a multiple of 16, got %zu at %p", cuts.need, workspace_bytes, workspace_dev);
        return NPAS_E_WORKSPACE;
    }
    a.q = q_dev; a.y = y_dev; a.lse = lse_dev; a.q_stride = q_stride; a.start = start_dev; a.length = length_dev;
    a.T = T; a.heads = heads; a.max_length = max_length; a.window = window; a.scale = scale;
    a.chunk = cuts.chunk; a.splits = cuts.splits; a.places = (int)plan.places;
    a.part = (float *)workspace_dev;
    a.part_stat = (float2 *)((uint8_t *)workspace_dev + cuts.stat_at);
    if (a.splits > 1)
        if (int rc = check_grid("chunk attention", (uint64_t)T * heads, join_threads(a.splits))) return rc;
    if (plan.groups) {
        AttentionArgs r{};
        r.c = a.c; r.q = a.q; r.y = a.y; r.lse = a.lse; r.q_stride = a.q_stride; r.start = a.start; r.length = a.length;
        r.T = T; r.heads = heads; r.max_length = max_length; r.window = window; r.scale = scale;
        r.chunk = a.chunk; r.splits = a.splits; r.waves = cuts.waves; r.places = a.places;
        r.part = a.part; r.part_stat = a.part_stat;
        if (int rc = launch_short_runs(dt, r, plan.groups, hip_stream)) return rc;
    } else if (int rc = launch_chunk_attention(dt, a, hip_stream)) return rc;
    return a.splits > 1 ? launch_chunk_join(dt, a, hip_stream) : NPAS_OK;
}

} // extern "C"
