// Expert FFN on 8-bit rows and weights (e4m3 with a power-of-two scale per 128 elements), a ragged grouped GEMM pair.
//
//   GEMM1  h = act(recv . W1^T [, recv . Wu^T]), quantised per 128 columns into packed rows
//   GEMM2  out = h . Wd^T, bf16
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies e4m3 operands with a power-of-two scale per row and 32 elements of K in the instruction
// itself, so the scales of a block of 128 cost no arithmetic.  The map of tiles is that of the bf16 kernels (ffn_tiles.h).
#include "ffn_tiles.h"
#include "fp8.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ExpertTable8 {
    const void *w1[MOE_MAX_LOCAL], *w_up[MOE_MAX_LOCAL], *w_down[MOE_MAX_LOCAL];
    const uint8_t *s1[MOE_MAX_LOCAL], *s_up[MOE_MAX_LOCAL], *s_down[MOE_MAX_LOCAL];
};
__device__ __forceinline__ float silu8(float a) { return a / (1.f + __expf(-a)); }
__device__ __forceinline__ float gelu8(float a) {
    const float u = 0.7978845608028654f * (a + 0.044715f * a * a * a);
    return a / (1.f + __expf(-2.f * u));
}
template <int EPI> __device__ __forceinline__ float activation8(float a, float b) {
    if (EPI == EPI_SILU) return silu8(a);
    if (EPI == EPI_GELU) return gelu8(a);
    if (EPI == EPI_SWIGLU) return silu8(a) * b;
    return a;
}

// 64 rows x 128 output columns per block; the 4 waves share the columns.  Operands straight from memory: lane (r = lane % 32,
// half = lane / 32) holds 32 consecutive bytes of row r; a k-step is 64, a scale holds for two.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTable8 tab, int which0, int which1, int N, int K,
                                                       void* __restrict__ C, int ldc) {
    const int tile = blockIdx.y;
    if (tile >= *m.n_tiles) return;
    __shared__ uint32_t amax_of[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, half = lane >> 5;
    const int row0 = m.row0[tile], nrows = m.nrows[tile], ex = m.expert[tile];
    const int32_t* rel = m.gather[tile] ? m.rel + (size_t)tile * kRelPitch : nullptr;
    const int n0 = blockIdx.x * 128, n = n0 + wave * 32;     // N is a multiple of 128
    size_t row[2];
    for (int i = 0; i < 2; ++i) {
        const int q = min(32 * i + r, nrows - 1);
        row[i] = (size_t)row0 + (rel ? rel[q] : q);
    }
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) for (int j = 0; j < 2; ++j) for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const char* b[2];
    const uint8_t* bs[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int which = j == 0 ? which0 : which1;
        b[j] = reinterpret_cast<const char*>(which == 0 ? tab.w1[ex] : which == 1 ? tab.w_up[ex] : tab.w_down[ex]) + (size_t)(n + r) * K + half * 32;
        bs[j] = (which == 0 ? tab.s1[ex] : which == 1 ? tab.s_up[ex] : tab.s_down[ex]) + (size_t)(n0 / 128) * (K / 128);
    }
    for (int k = 0; k < K; k += 64) {
        i32x8 av[2], bv[2];
        int sa[2], sb[2];
        for (int i = 0; i < 2; ++i) {
            av[i] = *reinterpret_cast<const i32x8*>(A + row[i] * lda + k + half * 32);
            sa[i] = A[row[i] * lda + K + k / 128];
        }
        for (int j = 0; j < (EPI == EPI_SWIGLU ? 2 : 1); ++j) {
            bv[j] = *reinterpret_cast<const i32x8*>(b[j] + k);
            sb[j] = bs[j][k / 128];
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < (EPI == EPI_SWIGLU ? 2 : 1); ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv[j], av[i], acc[i][j], 0, 0, 0, sb[j], 0, sa[i]);
    }
    // lane: row 32 i + r, columns n + 8 (e / 4) + 4 half + e % 4
    if (EPI == EPI_PLAIN) {
        for (int i = 0; i < 2; ++i) {
            if (32 * i + r >= nrows) continue;
            for (int e = 0; e < 16; e += 4) {
                uint2 q = make_uint2(f32_to_bf16_bits(acc[i][0][e]) | f32_to_bf16_bits(acc[i][0][e + 1]) << 16,
                                     f32_to_bf16_bits(acc[i][0][e + 2]) | f32_to_bf16_bits(acc[i][0][e + 3]) << 16);
                *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(C) + row[i] * ldc + n + 2 * e + 4 * half) = q;
            }
        }
        return;
    }
    for (int i = 0; i < 2; ++i) {
        uint32_t most = 0;
        for (int e = 0; e < 16; ++e) {
            acc[i][0][e] = activation8<EPI>(acc[i][0][e], EPI == EPI_SWIGLU ? acc[i][1][e] : 0.f);
            most = max(most, abs_bits(acc[i][0][e]));
        }
        most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
        if (half == 0) amax_of[wave][32 * i + r] = most;
    }
    __syncthreads();
    uint8_t* h = reinterpret_cast<uint8_t*>(C);
    for (int i = 0; i < 2; ++i) {
        const int q = 32 * i + r;
        if (q >= nrows) continue;
        const uint32_t most = max(max(amax_of[0][q], amax_of[1][q]), max(amax_of[2][q], amax_of[3][q]));
        const bool bad = fp8_block_is_nan(most);
        const uint32_t sb = bad ? 127u : fp8_scale_byte(most);
        const float inv = fp8_inverse_scale(sb);
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<uint32_t*>(h + row[i] * ldc + n + 2 * e + 4 * half) =
                bad ? 0x7f7f7f7fu : fp8_pack4(acc[i][0][e], acc[i][0][e + 1], acc[i][0][e + 2], acc[i][0][e + 3], inv);
        if (wave == 0 && half == 0) h[row[i] * ldc + N + n0 / 128] = (uint8_t)sb;
    }
}

template <int EPI>
int launch_fp8(const void* A, const TileMap& m, const ExpertTable8& tab, int which0, int which1, int N, int K, void* C, int ldc, int R, int nseg, hipStream_t st) {
    hipLaunchKernelGGL((gemm_fp8_kernel<EPI>), dim3(N / 128, max_tiles_of(R, 64, nseg)), dim3(256), 0, st, reinterpret_cast<const uint8_t*>(A), (int)fp8_row_bytes(K), m, tab,
                       which0, which1, N, K, C, ldc);
    MOE_LAUNCH_CHECK("gemm_fp8_kernel");
    return MOE_OK;
}

bool sizes_ok(int H, int F) { return H > 0 && F > 0 && H % FP8_BLOCK == 0 && F % FP8_BLOCK == 0 && (size_t)H * F <= 0xFFFFFFFFull; }

}  // namespace

extern "C" size_t moe_ffn_fp8_workspace_bytes(int32_t R_max, int32_t H, int32_t F, int32_t act) {
    if (R_max < 0 || !sizes_ok(H, F) || act < 0 || act > 2) return 0;
    return tilemap_bytes(R_max) + align256((size_t)R_max * fp8_row_bytes(F)) + 256;
}

extern "C" int moe_expert_ffn_fp8(const void* recv, int32_t R, const int32_t* seg_offset, const int32_t* seg_expert, int32_t nseg,
                                  const moe_expert_w8* experts, int32_t n_local, int32_t H, int32_t F, int32_t act, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (!recv || !seg_offset || !seg_expert || !experts || !out || !workspace) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_fp8: NULL argument");
    if (R < 0 || nseg < 0 || H <= 0 || F <= 0) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_fp8: negative size");
    if (act < 0 || act > 2) return moe_set_error(MOE_EDTYPE, "moe_expert_ffn_fp8: unknown act %d", act);
    if (n_local < 1 || n_local > MOE_MAX_LOCAL || nseg > kMaxSeg)
        return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_fp8: need 1 <= n_local <= %d and nseg <= %d", MOE_MAX_LOCAL, kMaxSeg);
    if (!sizes_ok(H, F)) return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_fp8: H and F must be multiples of 128, weight matrices below 4 GiB");
    if (!aligned16(recv) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return moe_set_error(MOE_EALIGN, "moe_expert_ffn_fp8: recv/out need 16-byte, workspace 256-byte alignment");
    if (workspace_bytes < moe_ffn_fp8_workspace_bytes(R, H, F, act))
        return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_fp8: workspace too small (%zu < %zu)", workspace_bytes, moe_ffn_fp8_workspace_bytes(R, H, F, act));
    ExpertTable8 tab;
    for (int e = 0; e < n_local; ++e) {
        const moe_expert_w8& w = experts[e];
        if (!w.w1 || !w.w_down || !w.s1 || !w.s_down || (act == MOE_ACT_SWIGLU && (!w.w_up || !w.s_up)))
            return moe_set_error(MOE_EINVAL, "moe_expert_ffn_fp8: expert %d has a NULL weight or scale", e);
        if (!aligned16(w.w1) || !aligned16(w.w_down) || !aligned16(w.w_up))
            return moe_set_error(MOE_EALIGN, "moe_expert_ffn_fp8: expert %d weights must be 16-byte aligned", e);
        tab.w1[e] = w.w1; tab.w_up[e] = w.w_up; tab.w_down[e] = w.w_down;
        tab.s1[e] = w.s1; tab.s_up[e] = w.s_up; tab.s_down[e] = w.s_down;
    }
    if (R == 0 || nseg == 0) return MOE_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const int ldh = (int)fp8_row_bytes(F);
    void* const h = reinterpret_cast<char*>(workspace) + tilemap_bytes(R);
    const int gather = 1;
    MapJobs jobs = {};
    jobs.job[0] = jobs.job[1] = MapJob{64, max_tiles_of(R, 64, nseg), tilemap_at(workspace, R)};
    if (nseg <= kSmallMapSegs) {
        const int blocks = std::min(64, (R / 64 + std::min(nseg, n_local) + 3) / 4);
        hipLaunchKernelGGL(tilemap_small_kernel<false>, dim3(blocks, 1), dim3(256), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
    } else {
        hipLaunchKernelGGL(tilemap_kernel, dim3(1), dim3(kMapThreads), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
    }
    MOE_LAUNCH_CHECK("tilemap_kernel");
    const TileMap& m = jobs.job[0].m;
    int rc;
    if (act == MOE_ACT_SWIGLU) rc = launch_fp8<EPI_SWIGLU>(recv, m, tab, 0, 1, F, H, h, ldh, R, nseg, st);
    else if (act == MOE_ACT_GELU_MLP) rc = launch_fp8<EPI_GELU>(recv, m, tab, 0, 0, F, H, h, ldh, R, nseg, st);
    else rc = launch_fp8<EPI_SILU>(recv, m, tab, 0, 0, F, H, h, ldh, R, nseg, st);
    if (rc != MOE_OK) return rc;
    return launch_fp8<EPI_PLAIN>(h, m, tab, 2, 2, H, F, out, H, R, nseg, st);
}
