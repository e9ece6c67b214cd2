// 8-bit floats of a cache (e4m3: sign, four exponent bits with bias 7, three mantissa bits) with the power of two of their block, and 16-bit numbers.
#pragma once
#include "device_util.h"

namespace npas {

// Exponents that a scale may have: the smallest and the largest number times it (240 of it at the upper end) are numbers of the 16-bit type,
// bf16 ones without its denormals, so that what is read is what was written.
template <int DT> struct Scale8 {
    static constexpr int least = DT == NPAS_BF16 ? -110 : -15, most = DT == NPAS_BF16 ? 120 : 8;
};

// Two of a word's four numbers times 2^(byte - 127) as 16-bit numbers, exact.
template <int DT, bool HI> __device__ __forceinline__ uint32_t from_e4m3x2(uint32_t codes, uint32_t byte)
{
    const float scale = __uint_as_float(byte << 23);
    if constexpr (DT == NPAS_BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HI));
}
template <int DT> __device__ __forceinline__ uint4 from_e4m3x8(uint2 codes, uint32_t byte)
{
    return make_uint4(from_e4m3x2<DT, false>(codes.x, byte), from_e4m3x2<DT, true>(codes.x, byte), from_e4m3x2<DT, false>(codes.y, byte),
                      from_e4m3x2<DT, true>(codes.y, byte));
}

// The top bits of those of a word's four codes that stand for NaN: by the code or by the scale byte.
__device__ __forceinline__ uint32_t nan_codes(uint32_t codes, uint32_t byte)
{
    const uint32_t n = ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return byte == 255 ? 0x80808080u : n;
}

// The scale byte of a block whose largest magnitude has the bits `top` (of fp32 without the sign; a NaN's are the largest).
template <int DT> __device__ __forceinline__ uint32_t scale8_of(uint32_t top)
{
    if (top >= 0x7f800000u) return 255;
    // top = f 2^E with 1 <= f < 2 is at most 448 2^e = 1.75 2^(e + 8) from e = E - 8 on, or from E - 7 where f is above 1.75
    const int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
    return (uint32_t)(min(max(e, Scale8<DT>::least), Scale8<DT>::most) + 127);
}
// Eight numbers of a block with that scale byte as codes.
template <int DT> __device__ __forceinline__ uint2 to_e4m3x8(const float (&x)[8], uint32_t byte)
{
    typedef short s2 __attribute__((ext_vector_type(2)));
    if (byte == 255) return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
    const float scale = __uint_as_float(byte << 23), most = (byte == Scale8<DT>::most + 127 ? 240.f : 448.f) * scale;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = __builtin_amdgcn_fmed3f(x[k], -most, most);
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s2 c = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * k], y[4 * k + 1], scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * k + 2], y[4 * k + 3], scale, true);
        w[k] = __builtin_bit_cast(uint32_t, c);
    }
    return make_uint2(w[0], w[1]);
}

} // namespace npas
