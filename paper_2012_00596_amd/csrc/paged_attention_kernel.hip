// Attention of one new token a sequence over the paged cache: the launches.
#include "paged_attention_kernel.h"

namespace npas {

int launch_paged_attention(int dt, const AttentionArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int group = a.heads / a.c.kv_heads;
    const dim3 grid((unsigned)((size_t)a.c.sequences * a.splits * ((group + 15) / 16) * a.c.kv_heads));
    if (int rc = check_grid("paged attention", grid.x, 64 * a.waves)) return rc;
    if (a.splits > 1)
        if (int rc = check_grid("paged attention", (uint64_t)a.c.sequences * a.heads, join_threads(a.splits))) return rc;
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
    };
    if (dt == NPAS_BF16) pick(std::integral_constant<int, NPAS_BF16>{});
    else pick(std::integral_constant<int, NPAS_F16>{});
    if (int rc = launched("paged attention")) return rc;
    return a.splits > 1 ? launch_join("paged attention", dt, a, (uint64_t)a.c.sequences * a.heads, st) : NPAS_OK;
}

} // namespace npas
