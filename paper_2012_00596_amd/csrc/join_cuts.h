// The cuts' sums of attention over the paged cache, joined.
#pragma once
#include <type_traits>

#include "decoder_internal.h"
#include "device_util.h"
#include "weight_parts.h"

namespace npas {

// The tokens of sequence s that take part: [first, first + count).
__device__ __forceinline__ void token_range(const AttentionArgs &a, int s, int &first, int &count)
{
    const long room = (long)a.c.table_stride * a.c.page_size;
    int n = max(0, min(a.length[s], a.max_length));
    if (n > room) n = (int)room;
    first = a.window > 0 ? max(0, n - a.window) : 0;
    count = n - first;
}

// One workgroup a row, (sequence, head) or (token, head): the cuts' sums, rescaled to the largest maximum and added; LANES lanes hold a cut's row, four elements
// each, so that THREADS / LANES cuts are read side by side.  One wave for up to 16 cuts (2048 rows of two cuts: 3 us, with eight
// waves 8.5), eight for more (32 rows of 128 cuts 4.8 us; 512 cuts read one after the other by four waves 37).
// A chain of latencies for few rows; for many the bytes of the sums, head_dim floats a row and cut.
template <int DT, int LANES, int THREADS, typename Args> __global__ __launch_bounds__(THREADS) void paged_attention_join_kernel(Args a)
{
    constexpr bool RUNS = std::is_same_v<Args, ChunkArgs>;
    constexpr int SIDE = THREADS / LANES, WAVES = THREADS / 64;
    __shared__ float weight[THREADS], part[WAVES], total[WAVES];
    __shared__ __align__(16) float so[SIDE][LANES * 4];
    const int D = a.c.head_dim, tid = threadIdx.x, side = tid / LANES, d = tid % LANES * 4;
    const size_t row = blockIdx.x;
    int cuts = a.splits;
    if constexpr (RUNS) {
        const int token = (int)(row / a.heads);
        if (token < a.start[0] || token >= a.start[a.c.sequences]) return; // no sequence's
    } else {
        int first, count;
        token_range(a, blockIdx.x / a.heads, first, count);
        cuts = (int)(((uint32_t)count + (uint32_t)a.chunk - 1) / (uint32_t)a.chunk); // (count and chunk together pass 2^31)
    }
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
    weight[tid] = RUNS && x.x == -INFINITY ? -1.f : c; // (a run's row that a cut has no token of: nothing is written there but that)
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
            if (RUNS && k < 0.f) continue;
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
    if constexpr (RUNS) l *= 1.f / RunWeight<DT>::unit;
    if (tid == 0 && a.lse) a.lse[row] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// Joins `rows` rows of y: launches of single tokens (AttentionArgs) or of runs (ChunkArgs).
template <typename Args> int launch_join(const char *what, int dt, const Args &a, uint64_t rows, hipStream_t st)
{
    const unsigned joiners = join_threads(a.splits);
    auto pick = [&](auto dtc, auto lanesc) {
        constexpr int DT = decltype(dtc)::value, LANES = decltype(lanesc)::value;
        const dim3 grid((unsigned)rows), block(joiners);
        if (joiners == 64) hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, 64, Args>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, kMaxSplits, Args>), grid, block, 0, st, a);
    };
    auto width = [&](auto dtc) {
        if (a.c.head_dim <= 64) pick(dtc, std::integral_constant<int, 16>{});
        else if (a.c.head_dim <= 128) pick(dtc, std::integral_constant<int, 32>{});
        else pick(dtc, std::integral_constant<int, 64>{});
    };
    if (dt == NPAS_BF16) width(std::integral_constant<int, NPAS_BF16>{});
    else width(std::integral_constant<int, NPAS_F16>{});
    return launched(what);
}

} // namespace npas
