// Rows held in the registers of waves, 8 neighbouring elements a lane, for the kernels that norm them (norm.hip, block_norm.hip): loads, stores, sums and
// roundings in 64 bits.
#pragma once
#include "fp8.h"
#include "lanes.h"
#include <algorithm>

namespace {

constexpr int kNormMaxH = 32768;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// two numbers rounded to nearest even, NaN to NaN, by one instruction
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }

template <int DT> __device__ __forceinline__ void load8(const void* p, size_t i, float (&v)[8]) {
    if (DT == MOE_BF16) {
        const u32x4 q = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(p) + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[2 * j] = bf16_bits_to_f32(q[j] & 0xffffu); v[2 * j + 1] = __uint_as_float(q[j] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 q = *reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(p) + i + 4 * j);
#pragma unroll
            for (int t = 0; t < 4; ++t) v[4 * j + t] = __uint_as_float(q[t]);
        }
    }
}
// LATER: what is not read again soon leaves the caches to what is
template <int DT, bool LATER> __device__ __forceinline__ void store8(void* p, size_t i, const float (&v)[8], int n) {
    if (DT == MOE_BF16) {
        u32x4 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
        u32x4* const to = reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(p) + i);
        if (LATER) __builtin_nontemporal_store(q, to);
        else *to = q;
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (4 * j < n) {
                const u32x4 q = {__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3])};
                u32x4* const to = reinterpret_cast<u32x4*>(reinterpret_cast<float*>(p) + i + 4 * j);
                if (LATER) __builtin_nontemporal_store(q, to);
                else *to = q;
            }
    }
}
// f = d rounded to fp32, to be rounded on to bf16 or e4m3: where f may lie halfway between two of those or at the limit of a scale (all of which have 15 zero
// bits at the end) and d does not, f moves one unit towards d, so that both roundings together are one.  A wave in sixty takes the branch.
__device__ __forceinline__ float towards(float f, double d) {
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffu) != 0u) return f;
    if (f == 0.f || !(fabsf(f) <= 3.40282347e38f) || (double)f == d) return f;
    return __uint_as_float((d > (double)f) == (f > 0.f) ? u + 1u : u - 1u);
}
// 1 / sqrt(m): the hardware's estimate and two steps of Newton's method, each of which squares the error; 0 gives NaN
__device__ __forceinline__ double inverse_root(double m) {
    double y = __builtin_amdgcn_rsq(m);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = __builtin_fma(y * 0.5, __builtin_fma(-m * y, y, 1.0), y);
    return y;
}
// Rows per launch: of 2^32 threads and more only the number modulo 2^32 would run, with no error
constexpr int64_t kLaunchThreads = (int64_t)1 << 31;

}  // namespace
