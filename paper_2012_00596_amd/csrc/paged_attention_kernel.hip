// Attention of one new token a sequence over the paged cache: a split kernel that walks the tokens once with running maximum and
// sum, and a joining kernel for sequences that were cut over several workgroups.
#include "paged_attention_kernel.h"

namespace npas {

// One workgroup a (sequence, head): the cuts' sums, rescaled to the largest maximum and added; LANES lanes hold a cut's row, four elements
// each, so that THREADS / LANES cuts are read side by side.  One wave for up to 16 cuts (2048 rows of two cuts: 3 us, with eight
// waves 8.5), eight for more (32 rows of 128 cuts 4.8 us; 512 cuts read one after the other by four waves 37).
template <int DT, int LANES, int THREADS> __global__ __launch_bounds__(THREADS) void paged_attention_join_kernel(AttentionArgs a)
{
    constexpr int SIDE = THREADS / LANES, WAVES = THREADS / 64;
    __shared__ float weight[THREADS], part[WAVES], total[WAVES];
    __shared__ __align__(16) float so[SIDE][LANES * 4];
    const int s = blockIdx.x / a.heads, D = a.c.head_dim, tid = threadIdx.x, side = tid / LANES, d = tid % LANES * 4;
    const size_t row = blockIdx.x;
    int first, count;
    token_range(a, s, first, count);
    const int cuts = (int)(((uint32_t)count + (uint32_t)a.chunk - 1) / (uint32_t)a.chunk); // (count and chunk together pass 2^31)
    const float2 x = tid < cuts ? a.part_stat[row * a.splits + tid] : make_float2(-INFINITY, 0.f); // no more cuts than threads
    float m = x.x;
#pragma unroll
    for (int w = 32; w; w >>= 1) m = fmaxf(m, __shfl_xor(m, w));
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, part[w]);
    const float c = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
    float l = c * x.y;
    weight[tid] = c;
#pragma unroll
    for (int w = 32; w; w >>= 1) l += __shfl_xor(l, w);
    if ((tid & 63) == 0) total[tid >> 6] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) l += total[w];
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d < D)
#pragma unroll 4
        for (int i = side; i < cuts; i += SIDE) {
            const float k = weight[i];
            const float4 v = *reinterpret_cast<const float4 *>(a.part + (row * a.splits + i) * D + d);
            y.x += k * v.x, y.y += k * v.y, y.z += k * v.z, y.w += k * v.w;
        }
    *reinterpret_cast<float4 *>(&so[side][d]) = y;
    __syncthreads();
    for (int i = tid; i < D; i += THREADS) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < SIDE; ++k) sum += so[k][i];
        reinterpret_cast<uint16_t *>(a.y)[row * D + i] = to_storage<DT>(l != 0.f ? sum / l : 0.f);
    }
    if (tid == 0 && a.lse) a.lse[row] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

int launch_paged_attention(int dt, const AttentionArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int group = a.heads / a.c.kv_heads;
    const dim3 grid((unsigned)((size_t)a.c.sequences * a.splits * ((group + 15) / 16) * a.c.kv_heads));
    const unsigned joiners = a.splits <= 16 ? 64 : kMaxSplits; // threads of a workgroup that joins
    if (int rc = check_grid("paged attention", grid.x, 64 * a.waves)) return rc;
    if (a.splits > 1)
        if (int rc = check_grid("paged attention", (uint64_t)a.c.sequences * a.heads, joiners)) return rc;
    auto pick = [&](auto dtc) {
        constexpr int DT = decltype(dtc)::value;
        auto run = [&](auto ncc) {
            constexpr int NC = decltype(ncc)::value;
            auto form = [&](auto nwc) {
                constexpr int NW = decltype(nwc)::value;
                auto width = [&](auto e8c) {
                    constexpr bool E8 = decltype(e8c)::value;
                    if (a.c.head_dim == 32 * NC) hipLaunchKernelGGL((paged_attention_kernel<DT, NC, true, NW, E8>), grid, dim3(64 * NW), 0, st, a);
                    else hipLaunchKernelGGL((paged_attention_kernel<DT, NC, false, NW, E8>), grid, dim3(64 * NW), 0, st, a);
                };
                if (a.c.k_scale) width(std::true_type{});
                else width(std::false_type{});
            };
            if constexpr (NC <= 4) {
                if (a.waves == 8) return form(std::integral_constant<int, 8>{});
            }
            form(std::integral_constant<int, 4>{});
        };
        if (a.c.head_dim <= 64) run(std::integral_constant<int, 2>{});
        else if (a.c.head_dim <= 128) run(std::integral_constant<int, 4>{});
        else run(std::integral_constant<int, 8>{});
        if (a.splits == 1) return;
        auto join = [&](auto lanesc) {
            constexpr int LANES = decltype(lanesc)::value;
            const dim3 rows((unsigned)(a.c.sequences * a.heads));
            if (joiners == 64) hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, 64>), rows, dim3(joiners), 0, st, a);
            else hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, kMaxSplits>), rows, dim3(joiners), 0, st, a);
        };
        if (a.c.head_dim <= 64) join(std::integral_constant<int, 16>{});
        else if (a.c.head_dim <= 128) join(std::integral_constant<int, 32>{});
        else join(std::integral_constant<int, 64>{});
    };
    if (dt == NPAS_BF16) pick(std::integral_constant<int, NPAS_BF16>{});
    else pick(std::integral_constant<int, NPAS_F16>{});
    return launched("paged attention");
}

} // namespace npas
