// Microscaled 4-bit floats: rows to codes and scales and back, and the product of quantised activations and packed weights on the
// scaled matrix instructions.
#include <type_traits>

#include "mxfp4_internal.h"
#include "row_vectors.h"

namespace npas {

// A quarter of a block (8 elements) to its codes; the four lanes of a block are neighbours and agree on its scale byte.  The largest
// magnitude is compared as bits: a NaN is above an infinity, an infinity above every number.  v times 2^-e is exact (down to the smallest
// fp32 numbers), the conversion rounds to nearest, ties to the even code.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t e = top >> 23;
    scale = e == 255 ? 255u : e > 2 ? e - 2 : 0u;
    if (e == 255) return 0u;
    const float inv = __uint_as_float((254u - scale) << 23);
    uint32_t c = 0;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = __builtin_amdgcn_fmed3f(v[k] * inv, -6.f, 6.f);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[0], w[1], 1.f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[2], w[3], 1.f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[4], w[5], 1.f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[6], w[7], 1.f, 3);
    return c;
}

// Canonical rows: four lanes a block, 64 blocks of one row a workgroup.
template <int DT> __global__ __launch_bounds__(256) void mxfp4_quantize_kernel(QuantizeArgs a)
{
    const int row = blockIdx.x, b = blockIdx.y * 64 + (int)(threadIdx.x >> 2), part = threadIdx.x & 3, k0 = b * 32 + part * 8;
    float v[8];
    load8<DT>(a.x, (size_t)row * a.x_stride + k0, a.K - k0, v);
    uint32_t scale;
    const uint32_t c = encode8(v, scale);
    if (b >= a.blocks) return;
    reinterpret_cast<uint32_t *>(a.codes)[((size_t)row * a.blocks + b) * 4 + part] = c;
    if (part == 0) a.scales[(size_t)row * a.blocks + b] = (uint8_t)scale;
}

// Operand images: a wave takes one block of 16 rows, a workgroup a step of a tile.
template <int DT> __global__ __launch_bounds__(256) void mxfp4_quantize_images_kernel(QuantizeArgs a)
{
    const int step = blockIdx.x % a.steps, tile = blockIdx.x / a.steps, q = threadIdx.x >> 6, r = threadIdx.x >> 2 & 15, part = threadIdx.x & 3;
    const int row = tile * 16 + r, k0 = step * 128 + q * 32 + part * 8;
    float v[8];
    load8<DT>(a.x, (size_t)(row < a.rows ? row : 0) * a.x_stride + k0, row < a.rows ? a.K - k0 : 0, v);
    uint32_t scale;
    const uint32_t c = encode8(v, scale);
    reinterpret_cast<uint32_t *>(a.codes)[((size_t)tile * a.steps + step) * 256 + threadIdx.x] = c;
    if (part == 0) a.scales[(((size_t)tile * a.quads + (step >> 2)) * 64 + q * 16 + r) * 4 + (step & 3)] = (uint8_t)scale;
}

template <int DT> __global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(DequantizeArgs a)
{
    const int row = blockIdx.x, b = blockIdx.y * 64 + (int)(threadIdx.x >> 2), part = threadIdx.x & 3, k0 = b * 32 + part * 8;
    if (b >= a.blocks) return;
    const uint32_t c = reinterpret_cast<const uint32_t *>(a.codes)[((size_t)row * a.blocks + b) * 4 + part], s = a.scales[(size_t)row * a.blocks + b];
    const float unit = s == 255 ? __uint_as_float(0x7fc00000u) : s ? __uint_as_float(s << 23) : __uint_as_float(0x00400000u);
    float v[8];
#define NPAS_PAIR(i)                                                     \
    {                                                                    \
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, i); \
        v[2 * i] = p[0] * unit;                                          \
        v[2 * i + 1] = p[1] * unit;                                      \
    }
    NPAS_PAIR(0) NPAS_PAIR(1) NPAS_PAIR(2) NPAS_PAIR(3)
#undef NPAS_PAIR
    store8<DT>(a.y, (size_t)row * a.K + k0, a.K - k0, v);
}

// ---- product --------------------------------------------------------------------

typedef __attribute__((ext_vector_type(8))) int i32x8;
__device__ __forceinline__ i32x8 operand(uint4 v) { return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0}; }
// 16 x 16 x 128 of two 4-bit images; byte S of each lane's scale word is its block's scale.
template <int S> __device__ __forceinline__ f32x4 mfma_mx(uint4 a, uint32_t sa, uint4 b, uint32_t sb, f32x4 c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, 4, 4, S, (int)sa, S, (int)sb);
}

// Result register i of image j: row 4 q + i of the tile, output 64 group + 4 n + j: a lane stores four consecutive outputs of a row.
struct __attribute__((packed, aligned(2))) Words8 {
    uint32_t w[2];
};
struct __attribute__((packed, aligned(4))) Floats4 {
    float f[4];
};
template <int DT> __device__ __forceinline__ void store_outputs(const FcMxArgs &a, int row, int o, float v0, float v1, float v2, float v3)
{
    float v[4] = {v0, v1, v2, v3};
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = act_apply(v[j] + (a.bias && o + j < a.OUT ? a.bias[o + j] : 0.f), a.act);
    const size_t at = (size_t)row * a.OUT + o;
    if (o + 4 <= a.OUT) {
        if constexpr (DT == NPAS_F32) *reinterpret_cast<Floats4 *>(reinterpret_cast<float *>(a.y) + at) = Floats4{v[0], v[1], v[2], v[3]};
        else *reinterpret_cast<Words8 *>(reinterpret_cast<uint16_t *>(a.y) + at) = Words8{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (o + j < a.OUT) st_act<DT>(a.y, at + j, v[j]);
    }
}

// One wave a tile of 16 rows and a group of 64 outputs.
template <int DT> __global__ __launch_bounds__(64) void fc_mxfp4_kernel(FcMxArgs a)
{
    const int lane = threadIdx.x, group = blockIdx.x % a.groups, tile = blockIdx.x / a.groups;
    const uint4 *x = reinterpret_cast<const uint4 *>(a.x_images) + (size_t)tile * a.steps * 64 + lane;
    const uint4 *w = reinterpret_cast<const uint4 *>(a.w_images) + (size_t)group * a.steps * 256 + lane;
    f32x4 c[4] = {};
    for (int quad = 0; quad < a.quads; ++quad) {
        const uint32_t sx = a.x_scales[((size_t)tile * a.quads + quad) * 64 + lane];
        uint32_t sw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) sw[j] = a.w_scales[(((size_t)group * a.quads + quad) * 4 + j) * 64 + lane];
        auto step = [&](auto sc) {
            constexpr int S = decltype(sc)::value;
            const int s = quad * 4 + S;
            if (s >= a.steps) return;
            const uint4 xv = x[s * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = mfma_mx<S>(xv, sx, w[(s * 4 + j) * 64], sw[j], c[j]);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }
    const int n = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = tile * 16 + q * 4 + i;
        if (row < a.B) store_outputs<DT>(a, row, group * 64 + 4 * n, c[0][i], c[1][i], c[2][i], c[3][i]);
    }
}

// ---- launches -------------------------------------------------------------------

template <typename F> static int with_dtype(int dt, const char *what, F &&f)
{
    if (dt == NPAS_F32) f(std::integral_constant<int, NPAS_F32>{});
    else if (dt == NPAS_BF16) f(std::integral_constant<int, NPAS_BF16>{});
    else f(std::integral_constant<int, NPAS_F16>{});
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NPAS_OK;
    set_error("%s launch failed: %s", what, hipGetErrorString(e));
    return NPAS_E_HIP;
}

int launch_mxfp4_quantize(int dt, const QuantizeArgs &a, void *stream)
{
    const dim3 grid((unsigned)a.rows, (unsigned)((a.blocks + 63) / 64));
    return with_dtype(dt, "4-bit quantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_quantize_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

int launch_mxfp4_quantize_images(int dt, const QuantizeArgs &a, void *stream)
{
    const dim3 grid((unsigned)((a.rows + 15) / 16 * a.steps));
    return with_dtype(dt, "4-bit quantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_quantize_images_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

int launch_mxfp4_dequantize(int dt, const DequantizeArgs &a, void *stream)
{
    const dim3 grid((unsigned)a.rows, (unsigned)((a.blocks + 63) / 64));
    return with_dtype(dt, "4-bit dequantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_dequantize_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

int launch_fc_mxfp4(int dt, const FcMxArgs &a, void *stream)
{
    const dim3 grid((unsigned)(a.tiles * a.groups));
    return with_dtype(dt, "4-bit product", [&](auto dtc) {
        hipLaunchKernelGGL((fc_mxfp4_kernel<decltype(dtc)::value>), grid, dim3(64), 0, (hipStream_t)stream, a);
    });
}

} // namespace npas
