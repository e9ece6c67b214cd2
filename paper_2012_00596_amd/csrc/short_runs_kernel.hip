// Attention of short runs of new tokens over the paged cache: the kernel of single tokens with a run's rows as columns.
#include "paged_attention_kernel.h"

namespace npas {

int launch_short_runs(int dt, const AttentionArgs &a, int groups, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)((size_t)a.places * a.splits * a.c.kv_heads));
    if (int rc = check_grid("chunk attention", (uint64_t)a.places * a.splits * a.c.kv_heads, 64 * a.waves)) return rc;
    auto pick = [&](auto dtc) {
        constexpr int DT = decltype(dtc)::value;
        auto run = [&](auto ncc) {
            constexpr int NC = decltype(ncc)::value;
            auto form = [&](auto nwc, auto groupsc) {
                constexpr int NW = decltype(nwc)::value, G = decltype(groupsc)::value;
                auto width = [&](auto e8c) {
                    constexpr bool E8 = decltype(e8c)::value;
                    if (a.c.head_dim == 32 * NC) hipLaunchKernelGGL((paged_attention_kernel<DT, NC, true, NW, E8, G>), grid, dim3(64 * NW), 0, st, a);
                    else hipLaunchKernelGGL((paged_attention_kernel<DT, NC, false, NW, E8, G>), grid, dim3(64 * NW), 0, st, a);
                };
                if (a.c.k_scale) width(std::true_type{});
                else width(std::false_type{});
            };
            if constexpr (NC <= 4) {
                if (groups == 2) return form(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
                if (a.waves == 8) return form(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
            }
            form(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
        };
        if (a.c.head_dim <= 64) run(std::integral_constant<int, 2>{});
        else if (a.c.head_dim <= 128) run(std::integral_constant<int, 4>{});
        else run(std::integral_constant<int, 8>{});
    };
    if (dt == NPAS_BF16) pick(std::integral_constant<int, NPAS_BF16>{});
    else pick(std::integral_constant<int, NPAS_F16>{});
    return launched("chunk attention");
}

} // namespace npas
