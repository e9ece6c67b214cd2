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
// n < 8: the first n alone.
template <int DT> __device__ __forceinline__ void store8(void *p, size_t i, int n, const float (&v)[8])
{
    if (n >= 8) {
        if constexpr (DT == NPAS_F32) {
            Floats8 x;
#pragma unroll
            for (int k = 0; k < 8; ++k) x.f[k] = v[k];
            *reinterpret_cast<Floats8 *>(reinterpret_cast<float *>(p) + i) = x;
        } else {
            Words16 x;
#pragma unroll
            for (int k = 0; k < 4; ++k) x.w[k] = pack2<DT>(v[2 * k], v[2 * k + 1]);
            *reinterpret_cast<Words16 *>(reinterpret_cast<uint16_t *>(p) + i) = x;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < n) st_act<DT>(p, i + k, v[k]);
    }
}

} // namespace npas
