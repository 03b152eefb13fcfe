// 64-bit values across the lanes of a wave.
#pragma once
#include "common.h"

namespace {

// of the row of 16 lanes, rotated
template <int CTRL> __device__ __forceinline__ double ror(double v) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_update_dpp(0, (int)u.x, CTRL, 0xF, 0xF, true), __builtin_amdgcn_update_dpp(0, (int)u.y, CTRL, 0xF, 0xF, true)));
}
__device__ __forceinline__ double lane_of(double v, int l) {
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readlane(u.x, l), __builtin_amdgcn_readlane(u.y, l)));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += ror<0x128>(v); v += ror<0x124>(v); v += ror<0x122>(v); v += ror<0x121>(v);   // row_ror by 8, 4, 2, 1
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

}  // namespace
