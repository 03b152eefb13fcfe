// 8-bit rows (e4m3 with a power-of-two scale per 128 elements): layout and quantisation, shared by the kernels that write them.
#pragma once
#include "common.h"

#define FP8_BLOCK 128

__host__ __device__ static inline size_t fp8_row_bytes(int H) { return ((size_t)H + H / FP8_BLOCK + 127) & ~(size_t)127; }

// Lanes that hold 8 neighbouring elements each, 16 of them a block of 128: the largest |v| over the block as bits.  The order of the bits of
// non-negative floats is that of the numbers, and NaNs come last, so the integer maximum finds those too.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xF, 0xF, true));   // row_ror:8
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xF, 0xF, true));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x122, 0xF, 0xF, true));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x121, 0xF, 0xF, true));
    return m;
}

// Scale byte of a block whose largest |v| has these bits: smallest b with |v| <= 448 * 2^(b - 127).  448 = 1.75 * 2^8, so with |v| = m * 2^x
// it is x - 8 + 127, one more for m > 1.75, which the addition carries into the exponent.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t amax) { return (uint32_t)max((int)((amax + 0x1fffffu) >> 23) - 8, 1); }
__device__ __forceinline__ bool fp8_block_is_nan(uint32_t amax) { return amax >= 0x7f800000u; }
// 1 / 2^(b - 127), exact
__device__ __forceinline__ float fp8_inverse_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// four elements, rounded to nearest even by the conversion; |v| * inv <= 448, so nothing overflows
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d, float inv) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, p, true);
}
