// Attention of one new token a sequence over the paged cache.
#include <type_traits>

#include "decoder_internal.h"
#include "device_util.h"

namespace npas {

// One workgroup a (sequence, head): four waves take the tokens in turn, a lane four elements of the head; running maximum and sum per
// wave, joined at the end.
template <int DT> __global__ __launch_bounds__(256) void paged_attention_kernel(AttentionArgs a)
{
    __shared__ float sm[4], sl[4], so[4][256];
    const int s = blockIdx.x / a.heads, head = blockIdx.x - s * a.heads, kv = head / (a.heads / a.c.kv_heads), D = a.c.head_dim;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d0 = lane * 4;
    const long room = (long)a.c.table_stride * a.c.page_size;
    int n = max(0, min(a.length[s], a.max_length));
    if (n > room) n = (int)room;
    const int first = a.window > 0 ? max(0, n - a.window) : 0;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = d0 + k < D ? a.scale * ld_act<DT>(a.q, (size_t)s * a.q_stride + (size_t)head * D + d0 + k) : 0.f;
    for (int j = first + wave; j < n; j += 4) {
        const int column = j / a.c.page_size, page = a.c.table[(size_t)s * a.c.table_stride + column];
        if ((uint32_t)page >= (uint32_t)a.c.pages) continue;
        const size_t row = (((size_t)page * a.c.kv_heads + kv) * a.c.page_size + (j - column * a.c.page_size)) * D;
        float x = 0.f;
        if (d0 < D)
#pragma unroll
            for (int k = 0; k < 4; ++k) x = fmaf(q[k], ld_act<DT>(a.c.k, row + d0 + k), x);
#pragma unroll
        for (int w = 32; w; w >>= 1) x += __shfl_xor(x, w);
        const float top = fmaxf(m, x), c = m == -INFINITY ? 0.f : expf(m - top), p = x == -INFINITY ? 0.f : expf(x - top);
        l = l * c + p;
        if (d0 < D)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = o[k] * c + p * ld_act<DT>(a.c.v, row + d0 + k);
        m = top;
    }
    if (lane == 0) {
        sm[wave] = m;
        sl[wave] = l;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) so[wave][d0 + k] = o[k];
    __syncthreads();
    const int d = threadIdx.x;
    const float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    float sum = 0.f, y = 0.f;
    for (int w = 0; w < 4; ++w) {
        const float c = sm[w] == -INFINITY ? 0.f : expf(sm[w] - top);
        sum += c * sl[w];
        y += c * so[w][d];
    }
    if (d < D) st_act<DT>(a.y, ((size_t)s * a.heads + head) * D + d, sum != 0.f ? y / sum : 0.f);
    if (d == 0 && a.lse) a.lse[(size_t)s * a.heads + head] = sum != 0.f ? top + logf(sum) : -INFINITY;
}

int launch_paged_attention(int dt, const AttentionArgs &a, void *stream)
{
    const dim3 grid((unsigned)(a.c.sequences * a.heads)), block(256);
    if (dt == NPAS_BF16) hipLaunchKernelGGL((paged_attention_kernel<NPAS_BF16>), grid, block, 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((paged_attention_kernel<NPAS_F16>), grid, block, 0, (hipStream_t)stream, a);
    return launched("paged attention");
}

} // namespace npas
