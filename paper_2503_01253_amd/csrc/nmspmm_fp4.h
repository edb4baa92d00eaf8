// The 4-bit format of nmspmm_mx4.h on the device: codes of a sign and the
// magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1), 32 to a scale byte s that
// stands for 2^(s - 127).
//
// gfx950 converts both ways with the scale in the same instruction.  It takes
// the scale as a float and looks at its exponent field alone (sign and
// mantissa may hold anything; 0 counts as 2^-127, 255 gives NaN for every
// code), rounds to nearest, ties to even, and saturates at 6.
#ifndef NMSPMM_FP4_H
#define NMSPMM_FP4_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nmspmm_dtype.h"

namespace nmspmm {

constexpr uint32_t MX4_NAN = 255, MX4_LEAST = 2, MX4_MOST = 252;

// The float whose exponent field is byte I of four scales.
template <int I>
__device__ __forceinline__ float mx4_scale(uint32_t four)
{
    return __builtin_bit_cast(float, I < 3 ? four << (23 - 8 * I) : four >> 1);
}

typedef float mx4_f32x2 __attribute__((ext_vector_type(2)));

// The eight codes of a word, lowest first, as fp32 values.
__device__ __forceinline__ void mx4_values(uint32_t w, uint32_t scale, float (&x)[8])
{
    const float s = mx4_scale<0>(scale);
    mx4_f32x2 v;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), x[0] = v[0], x[1] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1), x[2] = v[0], x[3] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), x[4] = v[0], x[5] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3), x[6] = v[0], x[7] = v[1];
}

// The scale of a group whose largest magnitude has these bits (as an integer:
// an infinity or NaN above all else): the smallest 2^e with it <= 7 * 2^e.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top)
{
    if (top >= 0x7f800000u) return MX4_NAN;
    const int s = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);     // 7 * 2^e is 1.75 * 2^(e+2)
    return s < (int)MX4_LEAST ? MX4_LEAST : s > (int)MX4_MOST ? MX4_MOST : (uint32_t)s;
}

// Eight values of a group as a word of codes, lowest first.
__device__ __forceinline__ uint32_t mx4_codes(const float (&x)[8], uint32_t scale)
{
    if (scale == MX4_NAN) return 0;
    const float s = __builtin_bit_cast(float, scale << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

// An fp64 value as a float for the two functions above: towards zero, its last
// bit set where something was cut off, so that it lies on the same side of
// every border of theirs (which have a few leading bits only).
__device__ __forceinline__ float mx4_narrow(double x)
{
    const float f = (float)x;
    const double back = (double)f;
    if (back == x || x != x) return f;
    uint32_t bits = __builtin_bit_cast(uint32_t, f);
    if (fabs(back) > fabs(x)) --bits;
    return __builtin_bit_cast(float, bits | 1u);
}

}  // namespace nmspmm

#endif
