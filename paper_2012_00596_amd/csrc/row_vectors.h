// Eight consecutive elements as fp32 and back, at the alignment of one element: global loads and stores of 16 bytes need no more on
// this architecture.
#pragma once
#include "device_util.h"

namespace npas {

struct __attribute__((packed, aligned(2))) Words16 {
    uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) Floats8 {
    float f[8];
};
// n < 8: the first n, zeros behind them.
template <int DT> __device__ __forceinline__ void load8(const void *p, size_t i, int n, float (&v)[8])
{
    if (n >= 8) {
        if constexpr (DT == NPAS_F32) {
            const Floats8 x = *reinterpret_cast<const Floats8 *>(reinterpret_cast<const float *>(p) + i);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = x.f[k];
        } else {
            const Words16 x = *reinterpret_cast<const Words16 *>(reinterpret_cast<const uint16_t *>(p) + i);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = from_storage<DT>((uint16_t)(x.w[k >> 1] >> (k & 1) * 16));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < n ? ld_act<DT>(p, i + k) : 0.f;
    }
}
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
// n < 8: the first n alone.  Whole vectors leave as streams (non-temporal): what these kernels write is larger than an XCD's L2 or read by another
// XCD next (norm 4096 x 4096 38.0 -> 33.2 us, append of 8191 tokens 40.3 -> 32.8, 8192 x 4100 to 4 bits and back 36.0 -> 31.5; a norm and the
// 4-bit product that reads it 14.0 -> 14.3 at 16 rows, 29.8 -> 27.4 at 1024; streaming loads cost as much as they gain).
template <int DT> __device__ __forceinline__ void store8(void *p, size_t i, int n, const float (&v)[8])
{
    if (n >= 8) {
        if constexpr (DT == NPAS_F32) {
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const u32x4_any x = {__float_as_uint(v[k]), __float_as_uint(v[k + 1]), __float_as_uint(v[k + 2]), __float_as_uint(v[k + 3])};
                __builtin_nontemporal_store(x, reinterpret_cast<u32x4_any *>(reinterpret_cast<float *>(p) + i + k));
            }
        } else {
            const u32x4_any x = {pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7])};
            __builtin_nontemporal_store(x, reinterpret_cast<u32x4_any *>(reinterpret_cast<uint16_t *>(p) + i));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < n) st_act<DT>(p, i + k, v[k]);
    }
}
// BYTES of LDS, 16-byte aligned, as they are, streamed likewise.
template <int BYTES> __device__ __forceinline__ void store_vectors(uint8_t *p, const uint8_t *from)
{
#pragma unroll
    for (int k = 0; k < BYTES; k += 16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(from + k);
        const u32x4_any x = {v.x, v.y, v.z, v.w};
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4_any *>(p + k));
    }
}

} // namespace npas
