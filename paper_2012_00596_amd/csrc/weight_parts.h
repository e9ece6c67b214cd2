// Weights of a softmax, fp32, as 16-bit numbers for the matrix cores.
#pragma once
#include "device_util.h"

namespace npas {

// Attention of runs: a row's weight is UNIT of exp(score - the maximum in use), which follows the scores only where one exceeds it by 2^GROW.  bf16 weights are
// 1 at the most, so that sums of large values pass the end of fp32 no sooner than those of the attention of one token; fp16 ones, whose type ends at 2^-24
// below, 2^15.  (A factor of the exponential: an exponent moved by 8 or 11 would be rounded more coarsely.)
template <int DT> struct RunWeight {
    static constexpr float unit = DT == NPAS_BF16 ? 0x1p-8f : 0x1p11f, grow = DT == NPAS_BF16 ? 8.f : 4.f;
};

// Two 16-bit numbers below the weights a and b, next to them or nearly so; zero for zero.
template <int DT> __device__ __forceinline__ uint32_t below2(float a, float b)
{
    const uint32_t u = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u), w = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);
    if constexpr (DT == NPAS_BF16) return __builtin_amdgcn_perm(w, u, 0x07060302u);
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float(u), __uint_as_float(w)));
}

// The first 16-bit part of two weights, below them or equal, and what is left of them in their place: never zero where the weight is not (of fp16 weights, down
// to 2^-14), as an infinite value times a part of zero would be NaN.
template <int DT> __device__ __forceinline__ uint32_t part_below2(float &a, float &b)
{
    if constexpr (DT == NPAS_BF16) {
        // (what is taken away is smaller than the part by 2^-24 of it: the weight counts as larger by that, in the one instruction that the difference takes)
        const uint32_t u = __float_as_uint(a), w = __float_as_uint(b);
        constexpr float c = 1.f - 0x1p-24f;
        a = fmaf(__uint_as_float(u & 0xffff0000u), -c, a);
        b = fmaf(__uint_as_float(w & 0xffff0000u), -c, b);
        return __builtin_amdgcn_perm(w, u, 0x07060302u);
    } else {
        const uint32_t x = below2<DT>(a, b);
        a -= from_storage<DT>((uint16_t)x);
        b -= from_storage<DT>((uint16_t)(x >> 16));
        return x;
    }
}

} // namespace npas
