// C-ABI calls of the decoder-block operators: argument checks and launches.
#include "decoder_internal.h"

namespace npas {

bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
bool bad_stride(int64_t stride, int64_t row) { return stride < row || stride > (int64_t)1 << 40; }

int check_cache(const npas_kv_cache *c, const npas_kv_scales *scales, int heads, CacheArgs *out, int *dt)
{
    if (!c || !c->k_dev || !c->v_dev || !c->page_table_dev || (scales && (!scales->k_scale_dev || !scales->v_scale_dev))) {
        set_error("NULL argument (cache, its keys, values or page table, or a scale)");
        return NPAS_E_NULL;
    }
    const int rows = scales ? scales->dtype : c->dtype;
    if ((scales && c->dtype != NPAS_E4M3) || (rows != NPAS_BF16 && rows != NPAS_F16)) {
        if (scales) set_error("a cache with scales holds e4m3 for rows of bf16 or fp16, not storage type %d for rows of type %d", c->dtype, rows);
        else set_error("a cache holds bf16 or fp16, not storage type %d", c->dtype);
        return NPAS_E_DTYPE;
    }
    if (c->pages <= 0 || c->page_size <= 0 || c->kv_heads <= 0 || c->sequences <= 0 || c->table_stride <= 0 || c->head_dim <= 0 ||
        c->head_dim % 8 || c->head_dim > 256 || (double)c->pages * c->kv_heads * c->page_size > 2147483647.0) {
        set_error("bad cache: pages=%d kv_heads=%d page_size=%d head_dim=%d sequences=%d table_stride=%d", c->pages, c->kv_heads,
                  c->page_size, c->head_dim, c->sequences, c->table_stride);
        return NPAS_E_SHAPE;
    }
    if (heads <= 0 || heads % c->kv_heads || (double)heads * c->head_dim > 16777216.0 || (double)heads * c->sequences > 16777216.0) {
        set_error("%d heads over %d key heads of %d elements and %d sequences", heads, c->kv_heads, c->head_dim, c->sequences);
        return NPAS_E_SHAPE;
    }
    if (misaligned(c->k_dev, 16) || misaligned(c->v_dev, 16) || misaligned(c->page_table_dev, 4) ||
        (scales && (misaligned(scales->k_scale_dev, 16) || misaligned(scales->v_scale_dev, 16)))) {
        set_error("the caches and their scales need 16-byte alignment, the page table 4");
        return NPAS_E_SHAPE;
    }
    if (scales && c->head_dim % 16) {
        set_error("a cache of 8-bit floats takes head_dim in multiples of 16, not %d", c->head_dim);
        return NPAS_E_SHAPE;
    }
    *out = CacheArgs{c->k_dev, c->v_dev, c->page_table_dev, c->pages, c->page_size, c->kv_heads, c->head_dim, c->sequences, c->table_stride,
                     scales ? (uint8_t *)scales->k_scale_dev : nullptr, scales ? (uint8_t *)scales->v_scale_dev : nullptr};
    *dt = rows;
    return NPAS_OK;
}

// How a launch cuts the tokens.  A pair is a sequence's key head (with up to 16 of its query heads): one workgroup a pair and cut.
//   - Up to kSingle elements of keys a pair one cut: the joining launch takes longer to issue (1.6 to 2.4 us) than it saves (from call to call: 16
//     pairs of 777 tokens, head_dim 64, 8.0 us in one cut, 9.3 in seven; replayed from a graph 8.2 and 7.1; 128 pairs of 300 tokens,
//     head_dim 128, in a graph 7.2 and 9.9).
//   - In that case eight waves where every workgroup has a compute unit to itself (16 pairs of 777 tokens 8.7 us, with four 9.4); otherwise four,
//     two or three workgroups on a compute unit (512 pairs of up to 8192 tokens in one cut, in their order, 227 us, with eight waves 244).
//   - Longer ones in 512 workgroups (131071 tokens of 4 pairs 54 us, in 1024 workgroups 56), at least 128 tokens each (4096 tokens of 8 pairs
//     8.6 us, 256 each 10.3); and at most 2048, so that a long sequence in a ragged batch does not run alone at the end (512 pairs of
//     up to 8192 tokens 205 us, at most 1024 each 198 to 202); in 8-bit caches, whose cuts are read in half the time, at most 1024 (the same pairs 116 us, 2048
//     each 122, 512 each 118; 163 new tokens over 32 sequences of some 4096 65 us, 2048 each 67, 512 each 69).
// Cuts follow max_length, not the lengths, which are on the device: a launch for much longer sequences than it meets leaves compute units idle
// (8 pairs of 4096 tokens, head_dim 128, 8.7 us at max_length 4096, 11.7 at 32768, 25.5 at 131072; 128 pairs of 2048 26 us, 65 at 32768).
Cuts plan_cuts(const CacheArgs &c, long pairs, size_t rows, int max_length, int window)
{
    constexpr long kWorkgroups = 512, kLeast = 128, kSingle = 65536;
    const long kMost = c.k_scale ? 1024 : 2048;
    const long room = (long)c.table_stride * c.page_size, longest = max_length < room ? max_length : room;
    const long n = window > 0 && window < longest ? window : longest;
    Cuts k{};
    const bool single = n * c.head_dim <= kSingle;
    k.waves = single && c.head_dim <= 128 && pairs <= 256 ? 8 : 4;
    long chunk = (n * pairs + kWorkgroups - 1) / kWorkgroups;
    if (chunk > kMost) chunk = kMost;
    if (chunk < kLeast) chunk = kLeast;
    if (chunk < (n + kMaxSplits - 1) / kMaxSplits) chunk = (n + kMaxSplits - 1) / kMaxSplits;
    if (single) chunk = n;
    chunk = (chunk + 127) / 128 * 128;
    k.chunk = (int)chunk;
    k.splits = (int)((n + chunk - 1) / chunk);
    // the most cuts that any window can lead to: one where the longest length is one cut; otherwise each has kLeast tokens, and kMost or the
    // pair's share of the workgroups
    const long share = (kWorkgroups + pairs - 1) / pairs, capped = (longest + kMost - 1) / kMost;
    long most = (longest + kLeast - 1) / kLeast;
    if (most > (share > capped ? share : capped)) most = share > capped ? share : capped;
    if (most > kMaxSplits) most = kMaxSplits;
    if (longest * c.head_dim <= kSingle) most = 1;
    k.stat_at = rows * k.splits * c.head_dim * 4;
    if (k.splits > 1) k.need = rows * k.splits * (c.head_dim * 4 + 8);
    if (most > 1) k.bytes = rows * most * (c.head_dim * 4 + 8);
    return k;
}

} // namespace npas

using namespace npas;

namespace {

Cuts plan_cuts(const CacheArgs &c, int heads, int max_length, int window)
{
    const long group = heads / c.kv_heads;
    return npas::plan_cuts(c, (long)c.sequences * c.kv_heads * ((group + 15) / 16), (size_t)c.sequences * heads, max_length, window);
}
bool storage(int dt) { return dt == NPAS_F32 || dt == NPAS_BF16 || dt == NPAS_F16; }

int paged_attention(const npas_kv_cache *cache, const npas_kv_scales *scales, const void *q_dev, int64_t q_stride, void *y_dev, float *lse_dev,
                    int heads, const int32_t *length_dev, int max_length, int window, float scale, void *workspace_dev, size_t workspace_bytes,
                    void *hip_stream)
{
    AttentionArgs a{};
    int dt;
    if (int rc = check_cache(cache, scales, heads, &a.c, &dt)) return rc;
    if (!q_dev || !y_dev || !length_dev) {
        set_error("NULL argument (q=%p y=%p length=%p)", q_dev, y_dev, (const void *)length_dev);
        return NPAS_E_NULL;
    }
    if (max_length <= 0 || window < 0 || bad_stride(q_stride, (int64_t)heads * a.c.head_dim) || !(scale == scale)) {
        set_error("bad shape heads=%d max_length=%d window=%d q_stride=%lld scale=%g", heads, max_length, window, (long long)q_stride,
                  (double)scale);
        return NPAS_E_SHAPE;
    }
    if (misaligned(q_dev, 2) || misaligned(y_dev, 2) || misaligned(lse_dev, 4) || misaligned(length_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    const Cuts cuts = plan_cuts(a.c, heads, max_length, window);
    if ((double)a.c.sequences * cuts.splits * heads > 2147483647.0) {
        set_error("%d sequences x %d heads x %d cuts of max_length=%d are too many workgroups", a.c.sequences, heads, cuts.splits, max_length);
        return NPAS_E_SHAPE;
    }
    const size_t need = cuts.need;
    if (need && (!workspace_dev || workspace_bytes < need || misaligned(workspace_dev, 16))) {
        set_error("paged attention needs %zu bytes of workspace at a multiple of 16, got %zu at %p", need, workspace_bytes, workspace_dev);
        return NPAS_E_WORKSPACE;
    }
    a.q = q_dev; a.y = y_dev; a.lse = lse_dev; a.q_stride = q_stride; a.length = length_dev;
    a.heads = heads; a.max_length = max_length; a.window = window; a.scale = scale;
    a.chunk = cuts.chunk; a.splits = cuts.splits; a.waves = cuts.waves;
    a.part = (float *)workspace_dev;
    a.part_stat = (float2 *)((uint8_t *)workspace_dev + cuts.stat_at);
    return launch_paged_attention(dt, a, hip_stream);
}

} // namespace

extern "C" {

int npas_gated_residual_norm(const void *branch_dev, const void *h_dev, const void *gate_dev, int64_t gate_stride,
                             const float *post_weight_dev, const float *pre_weight_dev, float residual_scale, float eps,
                             void *h_out_dev, void *n_out_dev, int T, int D, npas_dtype dt, void *hip_stream)
{
    if (!h_dev || !h_out_dev || !pre_weight_dev != !n_out_dev) {
        set_error("NULL argument (h=%p h_out=%p pre_weight=%p n_out=%p)", h_dev, h_out_dev, (const void *)pre_weight_dev, n_out_dev);
        return NPAS_E_NULL;
    }
    if (!branch_dev && (gate_dev || post_weight_dev)) {
        set_error("NULL argument: a gate or a norm of a branch that is not there");
        return NPAS_E_NULL;
    }
    if (!storage(dt)) {
        set_error("unknown storage type %d", (int)dt);
        return NPAS_E_DTYPE;
    }
    if (T <= 0 || D <= 0 || D > 1 << 24 || (gate_dev && gate_stride != 0 && bad_stride(gate_stride, D)) || !(eps >= 0.f)) {
        set_error("bad shape T=%d D=%d gate_stride=%lld eps=%g", T, D, (long long)gate_stride, (double)eps);
        return NPAS_E_SHAPE;
    }
    const size_t e = (size_t)dtype_size(dt);
    if (misaligned(branch_dev, e) || misaligned(h_dev, e) || misaligned(gate_dev, e) || misaligned(h_out_dev, e) ||
        misaligned(n_out_dev, e) || misaligned(post_weight_dev, 4) || misaligned(pre_weight_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    NormArgs a{branch_dev, h_dev, gate_dev, post_weight_dev, pre_weight_dev, h_out_dev, n_out_dev, gate_stride, residual_scale, eps,
               (float)(1.0 / D), T, D};
    return launch_gated_residual_norm(dt, a, hip_stream);
}

int npas_kv_append(const npas_kv_cache *cache, const void *q_dev, int64_t q_stride, const void *k_dev, int64_t k_stride,
                   const void *v_dev, int64_t v_stride, void *q_out_dev, int T, int heads, const int32_t *sequence_dev,
                   const int32_t *position_dev, const float *cos_sin_dev, int positions, int rot_dim, npas_rotation kind,
                   void *hip_stream)
{
    AppendArgs a{};
    int dt;
    if (int rc = check_cache(cache, nullptr, heads, &a.c, &dt)) return rc;
    if (!k_dev || !v_dev || !position_dev || !q_dev != !q_out_dev || (rot_dim > 0 && !cos_sin_dev)) {
        set_error("NULL argument (q=%p q_out=%p k=%p v=%p position=%p cos_sin=%p)", q_dev, q_out_dev, k_dev, v_dev,
                  (const void *)position_dev, (const void *)cos_sin_dev);
        return NPAS_E_NULL;
    }
    const int64_t qrow = (int64_t)heads * a.c.head_dim, krow = (int64_t)a.c.kv_heads * a.c.head_dim;
    if (T <= 0 || rot_dim < 0 || rot_dim % 2 || rot_dim > a.c.head_dim || (rot_dim > 0 && positions <= 0) ||
        (q_dev && bad_stride(q_stride, qrow)) || bad_stride(k_stride, krow) || bad_stride(v_stride, krow) ||
        (kind != NPAS_ROTATE_HALVES && kind != NPAS_ROTATE_PAIRS)) {
        set_error("bad shape T=%d heads=%d rot_dim=%d positions=%d strides %lld %lld %lld rotation %d", T, heads, rot_dim, positions,
                  (long long)q_stride, (long long)k_stride, (long long)v_stride, (int)kind);
        return NPAS_E_SHAPE;
    }
    if (misaligned(q_dev, 2) || misaligned(k_dev, 2) || misaligned(v_dev, 2) || misaligned(q_out_dev, 2) ||
        misaligned(sequence_dev, 4) || misaligned(position_dev, 4) || misaligned(cos_sin_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    a.q = q_dev; a.k = k_dev; a.v = v_dev; a.q_out = q_out_dev;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.sequence = sequence_dev; a.position = position_dev; a.cos_sin = cos_sin_dev;
    a.T = T; a.heads = heads; a.positions = positions; a.rot_dim = rot_dim; a.pairs = kind == NPAS_ROTATE_PAIRS;
    return launch_kv_append(dt, a, hip_stream);
}

size_t npas_paged_attention_workspace_bytes(const npas_kv_cache *cache, int heads, int max_length)
{
    CacheArgs c;
    int dt;
    if (max_length <= 0 || check_cache(cache, nullptr, heads, &c, &dt)) return 0;
    return plan_cuts(c, heads, max_length, 0).bytes;
}

int npas_paged_attention(const npas_kv_cache *cache, const void *q_dev, int64_t q_stride, void *y_dev, float *lse_dev, int heads,
                         const int32_t *length_dev, int max_length, int window, float scale, void *workspace_dev,
                         size_t workspace_bytes, void *hip_stream)
{
    return paged_attention(cache, nullptr, q_dev, q_stride, y_dev, lse_dev, heads, length_dev, max_length, window, scale, workspace_dev,
                           workspace_bytes, hip_stream);
}

size_t npas_paged_attention8_workspace_bytes(const npas_kv_cache *cache, const npas_kv_scales *scales, int heads, int max_length)
{
    CacheArgs c;
    int dt;
    if (max_length <= 0 || !scales || check_cache(cache, scales, heads, &c, &dt)) return 0;
    return plan_cuts(c, heads, max_length, 0).bytes;
}

int npas_paged_attention8(const npas_kv_cache *cache, const npas_kv_scales *scales, const void *q_dev, int64_t q_stride, void *y_dev,
                          float *lse_dev, int heads, const int32_t *length_dev, int max_length, int window, float scale, void *workspace_dev,
                          size_t workspace_bytes, void *hip_stream)
{
    if (!scales) {
        set_error("NULL argument (scales)");
        return NPAS_E_NULL;
    }
    return paged_attention(cache, scales, q_dev, q_stride, y_dev, lse_dev, heads, length_dev, max_length, window, scale, workspace_dev,
                           workspace_bytes, hip_stream);
}

} // extern "C"
