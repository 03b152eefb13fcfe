// 8-bit integer rows with one fp32 scale each: layout and quantisation, shared by the kernels that write them.
//
// q = v / s rounded to the nearest whole number, ties to even, s = max |v| / 127 of the row, rounded to fp32, 2^-126 at least.  A packed row of H values
// is H bytes, the scale (4 bytes) and zeros up to a multiple of 128 bytes.  A row with an infinity or a NaN, or whose scale is none of fp32's numbers, is zeros with a NaN for a scale.
#pragma once
#include "common.h"

__host__ __device__ static inline size_t int8_row_bytes(int H) { return ((size_t)H + 4 + 127) & ~(size_t)127; }

struct Int8Scale { float s; double inverse; };               // inverse 0: a row of NaN
// of a row whose largest |v| is `most` (an infinity or NaN where the row holds one).  The quotient by 127 is a product with its remainder's added; the reciprocal of s is the
// hardware's estimate and two steps of Newton's method, each of which squares the error.
__device__ __forceinline__ Int8Scale int8_scale(double most) {
    const double q = most * (1.0 / 127.0);
    const float s = fmaxf((float)__builtin_fma(__builtin_fma(-127.0, q, most), 1.0 / 127.0, q), 0x1p-126f);   // (fmaxf of a NaN and a number is the number: told apart below)
    const bool fine = most < __builtin_huge_val() && s < __builtin_huge_valf();
    double r = __builtin_amdgcn_rcp((double)s);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(__builtin_fma(-(double)s, r, 1.0), r, r);
    return fine ? Int8Scale{s, r} : Int8Scale{__uint_as_float(0x7fc00000u), 0.0};
}
// v times the inverse is off v / s by 2^-52 of it, 1e-14 of the distance between two whole numbers.  Added to 1.5 * 2^52 it is rounded to a whole number, ties to even,
// whose two's complement the low bits of the sum are.
//
// TIES: v and s are numbers of 24 bits, whose quotient may be a half exactly.  Any other is 2^-26 at least from a half: v there and the halves of s are whole multiples of a quarter of
// the last bit of s.  Rounded to a multiple of 2^-30 first, the product is the half itself.  (A number of 8 bits is a half only of a scale of 8 bits; that is a power of two,
// whose inverse is exact, as the largest element divided by 127 has no run of sixteen like bits otherwise.  A number of 64 bits has been rounded itself.)
template <bool TIES> __device__ __forceinline__ uint32_t int8_pack4(double a, double b, double c, double d, double inverse) {
    auto q = [&](double v) {
        const double whole = TIES ? __builtin_fma(v, inverse, 0x1.8p22) + (0x1.8p52 - 0x1.8p22) : __builtin_fma(v, inverse, 0x1.8p52);
        return (uint32_t)__builtin_bit_cast(uint64_t, whole);
    };
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q(d), q(c), 0x0c0c0400u), __builtin_amdgcn_perm(q(b), q(a), 0x0c0c0400u), 0x05040100u);
}
