// Device helpers of the operators in MX4.
#pragma once

#include "nm_mx4_internal.h"
#include "nm_q8_device.h"

namespace nm {

// Scale byte of a block whose largest magnitude has these bits (a NaN's are larger than infinity's, those larger than any number's).
// 2^(floor(log2 a) - 2): the exponent field less 2.  Subnormal and zero blocks have the field 0.
__device__ inline unsigned mx4_scale(unsigned most)
{
    const unsigned ef = most >> 23;
    return ef >= 255 ? 255 : ef > 2 ? ef - 2 : 0;
}

// The power of two of a scale byte as fp32 (0: 2^-127, a subnormal; 255: NaN).
__device__ inline float mx4_power(unsigned b) { return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7fc00000u : b << 23); }

// Eight adjacent values as codes.  The instruction divides by the power of two, rounds to the nearest, ties to the even code, and stops at 6
// (compared with that for all bf16 values under the four scales around theirs and for 2 million fp32 values, ties and their neighbours
// among them).
__device__ inline unsigned mx4_codes(const float (&v)[8], unsigned scale)
{
    const float s = mx4_power(scale);
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], s, 3);
    return scale == 255 ? 0u : r;
}

// The values that eight codes stand for.  The conversion under the scale 1 is exact, and so is the product unless it leaves fp32's range.
__device__ inline void mx4_values(unsigned codes, unsigned scale, float (&v)[8])
{
    const float s = mx4_power(scale);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    v[0] = a[0] * s; v[1] = a[1] * s; v[2] = b[0] * s; v[3] = b[1] * s;
    v[4] = c[0] * s; v[5] = c[1] * s; v[6] = d[0] * s; v[7] = d[1] * s;
}

__device__ inline unsigned magnitude(float f) { return __float_as_uint(f) & 0x7fffffffu; }

}  // namespace nm
