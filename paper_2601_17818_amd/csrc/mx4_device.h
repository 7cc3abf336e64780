// Rows in 4 bits: groups of 32 neighbouring values share an exponent byte s, a value is code * 2^(s - 127), and a code is a
// sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (e2m1).  gfx950 converts two values an instruction either way, the power of two
// included; every value is a bf16, so nothing is rounded on the way back, and s = 255 gives NaN.
#pragma once

#include "device_utils.h"

namespace vitcop {

constexpr int MX4_GROUP = 32;

__device__ __forceinline__ float mx4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// the eight values of a dword of codes as four pairs of bf16, lowest code first
__device__ __forceinline__ u32x4 mx4_values(uint32_t codes, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// The exponent byte of a group whose largest magnitude has the bf16 bits `top`: the least exponent in [-125, 125] that
// leaves no magnitude above 7 steps.  (Up to 7, not 6: what saturates is then off by one step at most, like what lies
// between 4 and 6.  Signal to error of normal values 19.0 dB against 18.7 with 6 and 18.8 with 8.)  An infinity or a
// NaN among them: 255.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t top) {
    const int e = (int)(top >> 7) - 2 + ((top & 0x7F) > 0x60 ? 1 : 0);
    return top >= 0x7F80 ? 255u : (uint32_t)min(max(e, 2), 252);
}

// Eight of a group's values per lane, the group in four neighbouring lanes of a quad: its exponent byte (in all four) and
// this lane's codes (nearest, ties to the even code, above 6 to 6; 0 where the group is not finite).
__device__ __forceinline__ uint32_t mx4_codes(const uint4& x, uint32_t& exponent) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    auto mag = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
    const u16x2 t = __builtin_elementwise_max(__builtin_elementwise_max(mag(x.x), mag(x.y)),
                                              __builtin_elementwise_max(mag(x.z), mag(x.w)));
    int top = max((int)t.x, (int)t.y);
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0xB1, 0xF, 0xF, true));         // quad_perm 1 0 3 2
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0x4E, 0xF, 0xF, true));         // quad_perm 2 3 0 1
    exponent = mx4_exponent((uint32_t)top);
    const float scale = mx4_scale(exponent == 255u ? 127u : exponent);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.z), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.w), scale, 3);
    return exponent == 255u ? 0u : c;
}

}  // namespace vitcop
