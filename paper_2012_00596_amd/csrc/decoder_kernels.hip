// Decoder-block kernels that move rows once: norm / gate / residual / norm, and the append of rotated keys and values to a
// paged cache.
#include <type_traits>

#include "decoder_internal.h"
#include "row_vectors.h"

namespace npas {

// Sum over a row's WPR waves, the same in every lane; the waves' sums are added in their order.
template <int WPR> __device__ __forceinline__ float row_sum(float v, float *part)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) v += part[w];
    }
    return v;
}

// One pass over a row that stays in registers: WPR waves a row (four rows a workgroup where one wave is a row), NV vectors of 8
// elements a thread.  Memory bound: five tensors of 4096 x 4096 bf16 in 32 us (5.2 TB/s).  One vector a thread rather than two of half as
// many waves: 4096 x 4096 33.2 -> 31.8 us, 16 rows twice and a product between them 14.3 -> 12.7.
template <int DT, int NV, int WPR> __global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void gated_residual_norm_kernel(NormArgs a)
{
    constexpr int THREADS = 64 * WPR;
    __shared__ float part[2][WPR];
    const int row = WPR == 1 ? (int)(blockIdx.x * 4 + (threadIdx.x >> 6)) : (int)blockIdx.x;
    const int tid = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    if (WPR == 1 && row >= a.T) return;
    const size_t at = (size_t)row * a.D;
    float b[NV][8], h[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = (tid + j * THREADS) * 8, n = a.D - i;
        load8<DT>(a.h, at + i, n, h[j]);
        if (a.branch) load8<DT>(a.branch, at + i, n, b[j]);
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) b[j][k] = 0.f;
    }
    if (a.branch) {
        float r = 1.f;
        if (a.post) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) s = fmaf(b[j][k], b[j][k], s);
            r = 1.f / sqrtf(row_sum<WPR>(s, part[0]) * a.inv_d + a.eps);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = (tid + j * THREADS) * 8, n = a.D - i;
            float w[8], g[8];
            if (a.post) {
                load8<NPAS_F32>(a.post, i, n, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) b[j][k] *= r * w[k];
            }
            if (a.gate) {
                load8<DT>(a.gate, (size_t)row * a.gate_stride + i, n, g);
#pragma unroll
                for (int k = 0; k < 8; ++k) b[j][k] *= g[k];
            }
        }
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[j][k] = fmaf(a.scale, h[j][k], b[j][k]);
            s = fmaf(h[j][k], h[j][k], s);
        }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = (tid + j * THREADS) * 8;
        store8<DT>(a.h_out, at + i, a.D - i, h[j]);
    }
    if (!a.pre) return;
    const float r = 1.f / sqrtf(row_sum<WPR>(s, part[1]) * a.inv_d + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = (tid + j * THREADS) * 8, n = a.D - i;
        float w[8];
        load8<NPAS_F32>(a.pre, i, n, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] *= h[j][k] * r;
        store8<DT>(a.n_out, at + i, n, w);
    }
}

// Rows too long for registers: three walks over the row, the last of which forms h_out again and writes it (h_out may be h).
// Element by element: 1024 rows of 16392 in 105 us (1.6 TB/s as five tensors; of 16384, in registers, 26), 256 of 65536 in 178.
template <int DT> __global__ __launch_bounds__(1024) void gated_residual_norm_long_kernel(NormArgs a)
{
    __shared__ float part[2][16];
    const int row = blockIdx.x;
    const size_t at = (size_t)row * a.D;
    float r = 1.f;
    if (a.branch && a.post) {
        float s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += 1024) {
            const float b = ld_act<DT>(a.branch, at + i);
            s = fmaf(b, b, s);
        }
        r = 1.f / sqrtf(row_sum<16>(s, part[0]) * a.inv_d + a.eps);
    }
    auto value = [&](int i) {
        float b = a.branch ? ld_act<DT>(a.branch, at + i) : 0.f;
        if (a.branch && a.post) b *= r * a.post[i];
        if (a.branch && a.gate) b *= ld_act<DT>(a.gate, (size_t)row * a.gate_stride + i);
        return fmaf(a.scale, ld_act<DT>(a.h, at + i), b);
    };
    float q = 1.f;
    if (a.pre) {
        float s = 0.f;
        for (int i = threadIdx.x; i < a.D; i += 1024) {
            const float h = value(i);
            s = fmaf(h, h, s);
        }
        q = 1.f / sqrtf(row_sum<16>(s, part[1]) * a.inv_d + a.eps);
    }
    for (int i = threadIdx.x; i < a.D; i += 1024) {
        const float h = value(i);
        st_act<DT>(a.h_out, at + i, h);
        if (a.pre) st_act<DT>(a.n_out, at + i, a.pre[i] * (h * q));
    }
}

template <typename F> static void with_dtype(int dt, F &&f)
{
    if (dt == NPAS_F32) f(std::integral_constant<int, NPAS_F32>{});
    else if (dt == NPAS_BF16) f(std::integral_constant<int, NPAS_BF16>{});
    else f(std::integral_constant<int, NPAS_F16>{});
}

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NPAS_OK;
    set_error("%s launch failed: %s", what, hipGetErrorString(e));
    return NPAS_E_HIP;
}

int check_grid(const char *what, uint64_t workgroups, unsigned threads)
{
    if (workgroups * threads <= 0xffffffffu) return NPAS_OK;
    set_error("%s: %llu workgroups of %u threads are more than a launch can have", what, (unsigned long long)workgroups, threads);
    return NPAS_E_SHAPE;
}

int launch_gated_residual_norm(int dt, const NormArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const unsigned threads = a.D <= 2048 ? 256 : a.D <= 4096 ? 512 : 1024, workgroups = a.D <= 1024 ? ((unsigned)a.T + 3) / 4 : (unsigned)a.T;
    if (int rc = check_grid("gated residual norm", workgroups, threads)) return rc;
    with_dtype(dt, [&](auto dtc) {
        constexpr int DT = decltype(dtc)::value;
        const dim3 grid(workgroups), block(threads);
        if (a.D <= 512) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 1, 1>), grid, block, 0, st, a);
        else if (a.D <= 1024) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 2, 1>), grid, block, 0, st, a);
        else if (a.D <= 2048) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 1, 4>), grid, block, 0, st, a);
        else if (a.D <= 4096) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 1, 8>), grid, block, 0, st, a);
        else if (a.D <= 8192) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 1, 16>), grid, block, 0, st, a);
        else if (a.D <= 16384) hipLaunchKernelGGL((gated_residual_norm_kernel<DT, 2, 16>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((gated_residual_norm_long_kernel<DT>), grid, block, 0, st, a);
    });
    return launched("gated residual norm");
}

// ---- append to the paged cache -------------------------------------------------

// One workgroup a token.  A unit is eight consecutive elements (fewer at the end of a part): rotated in themselves (PAIRS), rotated with
// their partners rot_dim / 2 further on (halves), or copied (the rest of a rotated head, the values).  Queries first, then keys, then values.
// Memory bound: 8191 tokens of 32 + 8 + 8 heads of 128, bf16, 206 MB in 32.7 us (6.3 TB/s, what is written partly stays in the Infinity
// Cache); a decode step of 24 tokens 3.0 us.
// WHOLE: every part of a head is a multiple of eight long (the checks for fewer cost 5-50 %: 2000 tokens of 64 + 8 + 8 heads 15.0 -> 23.3 us).
template <int DT, bool PAIRS, bool WHOLE> __global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a)
{
    const int t = blockIdx.x, D = a.c.head_dim, half = a.rot_dim / 2;
    const int s = a.sequence ? a.sequence[t] : t, pos = a.position[t];
    const bool token = (uint32_t)s < (uint32_t)a.c.sequences && pos >= 0 && (a.rot_dim == 0 || pos < a.positions);
    const int column = token ? pos / a.c.page_size : 0, slot = token ? pos - column * a.c.page_size : 0;
    const int page = token && column < a.c.table_stride ? a.c.table[(size_t)s * a.c.table_stride + column] : -1;
    const bool stored = (uint32_t)page < (uint32_t)a.c.pages;
    const size_t row0 = stored ? (size_t)page * a.c.kv_heads * a.c.page_size + slot : 0; // cache row of the first head
    const float *cs = a.cos_sin + (size_t)(token ? pos : 0) * a.rot_dim;
    const int rotated_part = PAIRS ? a.rot_dim : half, rot_units = (rotated_part + 7) >> 3;
    const int head_units = rot_units + ((D - a.rot_dim + 7) >> 3), value_units = D >> 3;
    const int nq = a.q ? a.heads * head_units : 0, nk = a.c.kv_heads * head_units, nv = a.c.kv_heads * value_units;
    for (int u = threadIdx.x; u < nq + nk + nv; u += blockDim.x) {
        const bool is_q = u < nq, is_v = u >= nq + nk;
        if (!is_q && !stored) break;
        const int w = is_q ? u : is_v ? u - nq - nk : u - nq, per = is_v ? value_units : head_units, head = w / per, j = w - head * per;
        const bool rotated = !is_v && j < rot_units;
        const int d = is_v || rotated ? j * 8 : a.rot_dim + (j - rot_units) * 8, n = WHOLE ? 8 : min(8, (rotated ? rotated_part : D) - d);
        const void *src = is_q ? a.q : is_v ? a.v : a.k;
        void *dst = is_q ? a.q_out : is_v ? a.c.v : a.c.k;
        const size_t in = (size_t)t * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + (size_t)head * D + d;
        const size_t out = (is_q ? ((size_t)t * a.heads + head) * D : (row0 + (size_t)head * a.c.page_size) * D) + d;
        float x[8], p[8], c[8], z[8];
        load8<DT>(src, in, n, x);
        if (!token) { // only queries come here
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = p[k] = 0.f;
        } else if (PAIRS && rotated) { // n is even
            const int m = n >> 1;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float co = k < m ? cs[d / 2 + k] : 0.f, si = k < m ? cs[half + d / 2 + k] : 0.f, u0 = x[2 * k], u1 = x[2 * k + 1];
                x[2 * k] = u0 * co - u1 * si;
                x[2 * k + 1] = u1 * co + u0 * si;
            }
        } else if (rotated) {
            load8<DT>(src, in + half, n, p);
            load8<NPAS_F32>(cs, d, n, c);
            load8<NPAS_F32>(cs, half + d, n, z);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float u0 = x[k], u1 = p[k];
                x[k] = u0 * c[k] - u1 * z[k];
                p[k] = u1 * c[k] + u0 * z[k];
            }
        }
        store8<DT>(dst, out, n, x);
        if (!PAIRS && rotated) store8<DT>(dst, out + half, n, p);
    }
}

int launch_kv_append(int dt, const AppendArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    // as many waves as one pass over the token's units fills, up to four (8191 tokens of 1 + 1 + 1 heads of 64: 5.7 us, always four 10.0)
    const int head_units = ((a.pairs ? a.rot_dim : a.rot_dim / 2) + 7) / 8 + (a.c.head_dim - a.rot_dim + 7) / 8;
    const long units = (long)((a.q ? a.heads : 0) + a.c.kv_heads) * head_units + (long)a.c.kv_heads * (a.c.head_dim / 8);
    const dim3 grid((unsigned)a.T), block(units <= 64 ? 64 : units <= 128 ? 128 : units <= 192 ? 192 : 256);
    if (int rc = check_grid("cache append", grid.x, block.x)) return rc;
    auto pick = [&](auto dtc) {
        constexpr int DT = decltype(dtc)::value;
        const bool whole = a.rot_dim % (a.pairs ? 8 : 16) == 0;
        if (a.pairs && whole) hipLaunchKernelGGL((kv_append_kernel<DT, true, true>), grid, block, 0, st, a);
        else if (a.pairs) hipLaunchKernelGGL((kv_append_kernel<DT, true, false>), grid, block, 0, st, a);
        else if (whole) hipLaunchKernelGGL((kv_append_kernel<DT, false, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((kv_append_kernel<DT, false, false>), grid, block, 0, st, a);
    };
    if (dt == NPAS_BF16) pick(std::integral_constant<int, NPAS_BF16>{});
    else pick(std::integral_constant<int, NPAS_F16>{});
    return launched("cache append");
}

} // namespace npas
