// Root-mean-square norm with the residual's addition, and 8-bit rows of its result.
//
//   r = round(x + residual);  v = r / sqrt(mean r^2 + eps) * gamma;  y = round(v);  rows = v quantised per 128 elements
//
// One pass: a row lives in the registers of W waves (8 neighbouring elements per lane and chunk of 512) from its load to its stores, the
// sum of squares crosses lanes by data-parallel moves and, for W > 1, waves through LDS.  A block of 128 elements is 16 lanes of a chunk, so its
// largest element needs no LDS.  Bound by memory: x, residual once in, r, y, rows once out.
//
// The sum, the root and the products are 64 bits: a row's factor is one number, and its roundings would shift all elements of the row alike, to the
// neighbouring e4m3 number where they lie near the middle of two.  y and the packed rows are what the 64-bit v rounds to, not its fp32 number.  16384 rows of 2048 with residual 54.8 us (5.5 TB/s), 16 rows of 4096 4.1; with everything in fp32 57.2 and 4.2, with division and root
// by the library's functions 62 and 4.6.
#include "norm_rows.h"

namespace {

// W waves per row, CH chunks of 512 elements per wave (chunk c of wave w: elements (c W + w) 512 ...); a block is 4 / W rows, one for W >= 3.
template <int DT, int W, int CH>
__global__ __launch_bounds__((W < 3 ? 256 : 64 * W)) void norm_kernel(const void* x, const void* residual, const void* __restrict__ gamma, float eps, double inv_h, int T, int H,
                                                                      void* residual_out, void* y, uint8_t* __restrict__ rows, int pitch) {
    constexpr int WAVES = W < 3 ? 4 : W;
    __shared__ double part[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
    const int row = blockIdx.x * (WAVES / W) + wave / W;
    const bool live = row < T;                               // the same for a wave; a dead one still meets the barrier
    const size_t base = (size_t)(live ? row : T - 1) * H;
    float v[CH][8], g[CH][8];
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * W + w) * 512 + lane * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) { v[c][j] = 0.f; g[c][j] = 1.f; }
        if (i < H && gamma) {                                // beside the row's loads: one round trip for both
            if (DT == MOE_F32 && i + 8 > H) {
#pragma unroll
                for (int j = 0; j < 4; ++j) g[c][j] = reinterpret_cast<const float*>(gamma)[i + j];
            } else {
                load8<DT>(gamma, i, g[c]);
            }
        }
        if (i < H) {                                         // fp32 rows may end in the middle of a lane's 8
            if (DT == MOE_F32 && i + 8 > H) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[c][j] = reinterpret_cast<const float*>(x)[base + i + j];
                if (residual)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[c][j] += reinterpret_cast<const float*>(residual)[base + i + j];
            } else {
                load8<DT>(x, base + i, v[c]);
                if (residual) {
                    float q[8];
                    load8<DT>(residual, base + i, q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[c][j] += q[j];
                    if (DT == MOE_BF16)
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const uint32_t s = bf16_pair(v[c][j], v[c][j + 1]);
                            v[c][j] = bf16_bits_to_f32(s & 0xffffu);
                            v[c][j + 1] = __uint_as_float(s & 0xffff0000u);
                        }
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)v[c][j], (double)v[c][j], sum);
        }
    }
    sum = wave_sum(sum);
    if (W > 1) {
        if (lane == 0) part[wave] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < W; ++i) sum += part[wave / W * W + i];
    }
    if (!live) return;
    // (a sum beyond fp32 counts as infinite)
    const double inv = sum <= 3.4028234663852886e38 ? inverse_root(__builtin_fma(sum, inv_h, (double)eps)) : sum > 0.0 ? 0.0 : sum;
    uint8_t* const out = rows ? rows + (size_t)row * pitch : nullptr;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int chunk = c * W + w, i = chunk * 512 + lane * 8, n = H - i;
        if (chunk * 512 >= H) break;
        if (residual_out && n > 0) store8<DT, true>(residual_out, base + i, v[c], n);
        if (n > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double d = (double)v[c][j] * inv * (double)g[c][j];
                v[c][j] = towards((float)d, d);
                g[c][j] = DT == MOE_BF16 ? v[c][j] : (float)d;
            }
            if (y) store8<DT, false>(y, base + i, g[c], n);
        }
        if (out) {                                           // H is a multiple of 128: 16 lanes have a whole block or none
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[c][j]));
            m = max_of_16_lanes(m);
            const bool bad = fp8_block_is_nan(m);
            const uint32_t b = bad ? 127u : fp8_scale_byte(m);
            const float s = fp8_inverse_scale(b);
            if (n > 0) {
                uint2 q = make_uint2(fp8_pack4(v[c][0], v[c][1], v[c][2], v[c][3], s), fp8_pack4(v[c][4], v[c][5], v[c][6], v[c][7], s));
                if (bad) q = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
                *reinterpret_cast<uint2*>(out + i) = q;
            }
            // the four scale bytes of the chunk as one word; a block beyond H gives zero, as the padding is
            const uint32_t byte = n > 0 ? b : 0u;
            const uint32_t word = __builtin_amdgcn_readlane(byte, 0) | __builtin_amdgcn_readlane(byte, 16) << 8 | __builtin_amdgcn_readlane(byte, 32) << 16 |
                                  (uint32_t)__builtin_amdgcn_readlane(byte, 48) << 24;
            if (lane == 0) *reinterpret_cast<uint32_t*>(out + H + 4 * chunk) = word;
        }
    }
    if (out)
        for (int i = (H + 511) / 512 + w * 64 + lane; i < (pitch - H) / 4; i += W * 64) *reinterpret_cast<uint32_t*>(out + H + 4 * i) = 0u;
}

template <int DT, int W, int CH>
int launch_rows(const void* x, const void* residual, const void* gamma, float eps, int T, int H, void* residual_out, void* y, uint8_t* rows, hipStream_t st) {
    const int pitch = (int)fp8_row_bytes(H), most = (int)(kLaunchThreads / (64 * W));
    const size_t row = (size_t)H * (DT == MOE_BF16 ? 2 : 4);
    for (int64_t t = 0; t < T; t += most) {
        const int n = (int)std::min<int64_t>(most, T - t);
        auto at = [&](const void* p) { return p ? reinterpret_cast<char*>(const_cast<void*>(p)) + t * row : nullptr; };
        hipLaunchKernelGGL((norm_kernel<DT, W, CH>), dim3(W < 3 ? (n * W + 3) / 4 : n), dim3(W < 3 ? 256 : 64 * W), 0, st, at(x), at(residual), gamma, eps, 1.0 / H, n, H, at(residual_out),
                           at(y), rows ? rows + (size_t)t * pitch : nullptr, pitch);
        MOE_LAUNCH_CHECK("norm_kernel");
    }
    return MOE_OK;
}
template <int DT>
int launch_norm(const void* x, const void* residual, const void* gamma, float eps, int T, int H, void* residual_out, void* y, uint8_t* rows, hipStream_t st) {
    const int chunks = (H + 511) / 512;
#define MOE_NORM(W, CH) return launch_rows<DT, W, CH>(x, residual, gamma, eps, T, H, residual_out, y, rows, st)
    // a chunk per wave where a block holds the row: 16384 rows of 2048 with residual, in fp32, 56 us (two chunks per wave 61, four 70)
    if (chunks <= 1) MOE_NORM(1, 1);
    if (chunks <= 2) MOE_NORM(2, 1);
    if (chunks <= 3) MOE_NORM(3, 1);
    if (chunks <= 4) MOE_NORM(4, 1);
    if (chunks <= 6) MOE_NORM(6, 1);
    if (chunks <= 8) MOE_NORM(8, 1);
    if (chunks <= 12) MOE_NORM(12, 1);
    if (chunks <= 16) MOE_NORM(16, 1);
    if (chunks <= 32) MOE_NORM(16, 2);
    MOE_NORM(16, 4);
#undef MOE_NORM
}

}  // namespace

extern "C" size_t moe_fp8_row_bytes(int32_t H) { return H > 0 && H % FP8_BLOCK == 0 ? fp8_row_bytes(H) : 0; }

extern "C" int moe_norm_fp8(const void* x, const void* residual, const void* gamma, float eps, int32_t T, int32_t H, int32_t dtype,
                            void* residual_out, void* y, void* rows, void* stream) {
    if (T != 0 && (!x || (!residual_out && !y && !rows))) return moe_set_error(MOE_EINVAL, "moe_norm_fp8: NULL argument");
    if (T < 0 || H <= 0 || !(eps >= 0.f) || eps > 3.4e38f) return moe_set_error(MOE_EINVAL, "moe_norm_fp8: T >= 0, H > 0 and a finite eps >= 0 required");
    if (dtype != MOE_F32 && dtype != MOE_BF16) return moe_set_error(MOE_EDTYPE, "moe_norm_fp8: unknown dtype %d", dtype);
    if (H > kNormMaxH) return moe_set_error(MOE_ESHAPE, "moe_norm_fp8: H <= %d required", kNormMaxH);
    if (rows && H % FP8_BLOCK != 0) return moe_set_error(MOE_ESHAPE, "moe_norm_fp8: packed rows need H to be a multiple of 128");
    if (((size_t)H * elem_size(dtype)) % 16 != 0) return moe_set_error(MOE_EALIGN, "moe_norm_fp8: row size H*elem must be a multiple of 16 bytes");
    if (!aligned16(x) || !aligned16(residual) || !aligned16(gamma) || !aligned16(residual_out) || !aligned16(y) || !aligned16(rows))
        return moe_set_error(MOE_EALIGN, "moe_norm_fp8: arrays must be 16-byte aligned");
    if (y && y == residual_out) return moe_set_error(MOE_EINVAL, "moe_norm_fp8: y and residual_out are the same array");
    if (T == 0) return MOE_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return dtype == MOE_BF16 ? launch_norm<MOE_BF16>(x, residual, gamma, eps, T, H, residual_out, y, reinterpret_cast<uint8_t*>(rows), st)
                             : launch_norm<MOE_F32>(x, residual, gamma, eps, T, H, residual_out, y, reinterpret_cast<uint8_t*>(rows), st);
}
