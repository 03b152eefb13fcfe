// Gate with scores, a balance bias and groups of experts.
//
//   l = x . Wg^T;  s = softmax(l) or sigmoid(l);  c = s + bias;  the top_groups groups of the largest rank;  the k largest c in them
//
// Two kernels: logits on the matrix cores into the workspace, then a wave per token that scores and selects.
#include "common.h"
#include <cmath>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A wave per 16 tokens x 16 experts.  Lane (r = lane % 16, g = lane / 16) takes chunks of 16 bytes g, g + 4, ... of its token row
// and expert row: the order of the sum over H is free.
template <int DT>
__global__ __launch_bounds__(256) void gate_logits_kernel(const char* __restrict__ x, const char* __restrict__ wg, int T, int H, int E, float* __restrict__ logits) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = (blockIdx.x * 4 + wave) * 16, e0 = blockIdx.y * 16;
    if (t0 >= T) return;
    const int r = lane & 15, g = lane >> 4;
    const size_t pitch = (size_t)H * (DT == MOE_BF16 ? 2 : 4);
    const char* px = x + (size_t)min(t0 + r, T - 1) * pitch;
    const char* pw = wg + (size_t)min(e0 + r, E - 1) * pitch;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const u32x4 none = {0u, 0u, 0u, 0u};
    for (size_t at = g * 16; at < ((pitch + 63) & ~(size_t)63); at += 64) {
        const bool in = at < pitch;
        const u32x4 a = in ? *reinterpret_cast<const u32x4*>(pw + at) : none, b = in ? *reinterpret_cast<const u32x4*>(px + at) : none;
        if (DT == MOE_BF16) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(&a), *reinterpret_cast<const bf16x8*>(&b), acc, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
        }
    }
    if (t0 + r < T)                                          // lane: token r, experts 4 g .. 4 g + 3
        for (int i = 0; i < 4; ++i)
            if (e0 + 4 * g + i < E) logits[(size_t)(t0 + r) * E + e0 + 4 * g + i] = acc[i];
}

__device__ __forceinline__ float wave_max(float v) {
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

constexpr int kPerLane = MOE_MAX_E / 64;

// A wave per token; lane l looks after experts l, l + 64, ...
__global__ __launch_bounds__(256) void gate_select_kernel(const float* __restrict__ logits, const float* __restrict__ bias, moe_gate_rule rule, int T, int E, int k,
                                                          int renorm, int32_t* __restrict__ topk_idx, float* __restrict__ topk_w) {
    __shared__ float score[4][MOE_MAX_E], rank[4][MOE_MAX_E];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * 4 + wave;
    const bool live = t < T;
    const float* row = logits + (size_t)(live ? t : T - 1) * E;
    float s[kPerLane], c[kPerLane];
    for (int i = 0; i < kPerLane; ++i) s[i] = lane + 64 * i < E ? row[lane + 64 * i] : -INFINITY;
    if (rule.score == MOE_SCORE_SOFTMAX) {
        float m = -INFINITY, sum = 0.f;
        bool nan = false;
        for (int i = 0; i < kPerLane; ++i) { m = fmaxf(m, s[i]); nan |= s[i] != s[i]; }
        m = wave_max(m);
        for (int i = 0; i < kPerLane; ++i) { s[i] = lane + 64 * i < E ? expf(s[i] - m) : 0.f; sum += s[i]; }
        sum = wave_sum(sum);
        if (__any(nan)) sum = NAN;
        for (int i = 0; i < kPerLane; ++i) s[i] /= sum;
    } else {
        for (int i = 0; i < kPerLane; ++i) s[i] = 1.f / (1.f + expf(-s[i]));
    }
    for (int i = 0; i < kPerLane; ++i) {
        const int e = lane + 64 * i;
        c[i] = e < E ? (bias ? s[i] + bias[e] : s[i]) : -INFINITY;
        if (!(c[i] == c[i])) c[i] = -INFINITY;
        if (e < E) score[wave][e] = c[i];
    }
    __syncthreads();
    if (rule.top_groups < rule.n_groups) {
        const int size = E / rule.n_groups;
        for (int g = lane; g < rule.n_groups; g += 64) {
            float a = -INFINITY, b = -INFINITY;              // the two largest
            for (int i = 0; i < size; ++i) {
                const float v = score[wave][g * size + i];
                b = fmaxf(b, fminf(a, v));
                a = fmaxf(a, v);
            }
            float r = rule.group_rank == MOE_GROUP_TOP2 && size > 1 ? a + b : a;
            rank[wave][g] = r == r ? r : -INFINITY;
        }
        __syncthreads();
        for (int i = 0; i < kPerLane; ++i) {
            const int e = lane + 64 * i;
            if (e >= E) continue;
            const int mine = e / size;
            int before = 0;
            for (int g = 0; g < rule.n_groups; ++g) before += rank[wave][g] > rank[wave][mine] || (rank[wave][g] == rank[wave][mine] && g < mine);
            if (before >= rule.top_groups) c[i] = -INFINITY;
        }
    }
    if (!live) return;
    float my_w = 0.f, sum = 0.f;
    int my_idx = -1;
    for (int j = 0; j < k; ++j) {
        float best = -INFINITY;
        int at = 0x7fffffff;
        for (int i = 0; i < kPerLane; ++i)
            if (c[i] > best) { best = c[i]; at = lane + 64 * i; }
        for (int o = 32; o > 0; o >>= 1) {
            const float ob = __shfl_xor(best, o, 64);
            const int oa = __shfl_xor(at, o, 64);
            if (ob > best || (ob == best && oa < at)) { best = ob; at = oa; }
        }
        if (best == -INFINITY) break;
        float w = 0.f;
        for (int i = 0; i < kPerLane; ++i)
            if (at == lane + 64 * i) { w = s[i]; c[i] = -INFINITY; }
        w = __shfl(w, at & 63, 64);
        sum += w;
        if (lane == j) { my_w = w; my_idx = at; }
    }
    if (lane < k) {
        topk_idx[(size_t)t * k + lane] = my_idx;
        topk_w[(size_t)t * k + lane] = (renorm ? (sum > 0.f ? my_w / sum : 0.f) : my_w) * rule.scale;
    }
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace

extern "C" size_t moe_route_grouped_workspace_bytes(const moe_ctx* ctx) {
    return ctx ? align256((size_t)ctx->s.T * ctx->s.E * sizeof(float)) : 0;
}

extern "C" int moe_route_grouped(moe_ctx* ctx, const void* x, const void* Wg, const moe_gate_rule* rule, const float* select_bias,
                                 int32_t* topk_idx, float* topk_w, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx || !x || !Wg || !rule || !topk_idx || !topk_w || !workspace) return moe_set_error(MOE_EINVAL, "moe_route_grouped: NULL argument");
    const moe_shape& s = ctx->s;
    if (rule->score != MOE_SCORE_SOFTMAX && rule->score != MOE_SCORE_SIGMOID) return moe_set_error(MOE_EINVAL, "moe_route_grouped: unknown score %d", rule->score);
    if (rule->group_rank != MOE_GROUP_MAX && rule->group_rank != MOE_GROUP_TOP2) return moe_set_error(MOE_EINVAL, "moe_route_grouped: unknown group_rank %d", rule->group_rank);
    if (rule->n_groups < 1 || rule->top_groups < 1) return moe_set_error(MOE_EINVAL, "moe_route_grouped: n_groups and top_groups must be positive");
    if (!std::isfinite(rule->scale)) return moe_set_error(MOE_EINVAL, "moe_route_grouped: scale must be finite");
    if (s.E % rule->n_groups != 0 || rule->top_groups > rule->n_groups || rule->top_groups * (s.E / rule->n_groups) < s.k)
        return moe_set_error(MOE_ESHAPE, "moe_route_grouped: %d groups, %d kept, do not fit E=%d, k=%d", rule->n_groups, rule->top_groups, s.E, s.k);
    if (!aligned16(x) || !aligned16(Wg) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return moe_set_error(MOE_EALIGN, "moe_route_grouped: x, Wg need 16-byte, workspace 256-byte alignment");
    if (workspace_bytes < moe_route_grouped_workspace_bytes(ctx))
        return moe_set_error(MOE_ESHAPE, "moe_route_grouped: workspace too small (%zu < %zu)", workspace_bytes, moe_route_grouped_workspace_bytes(ctx));
    ctx->rank_src = nullptr;                                 // new indices: no ranks to reuse
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    float* const logits = reinterpret_cast<float*>(workspace);
    const dim3 grid((s.T + 63) / 64, (s.E + 15) / 16);
    const char *px = reinterpret_cast<const char*>(x), *pw = reinterpret_cast<const char*>(Wg);
    if (s.dtype == MOE_BF16) hipLaunchKernelGGL((gate_logits_kernel<MOE_BF16>), grid, dim3(256), 0, st, px, pw, s.T, s.H, s.E, logits);
    else hipLaunchKernelGGL((gate_logits_kernel<MOE_F32>), grid, dim3(256), 0, st, px, pw, s.T, s.H, s.E, logits);
    MOE_LAUNCH_CHECK("gate_logits_kernel");
    hipLaunchKernelGGL(gate_select_kernel, dim3((s.T + 3) / 4), dim3(256), 0, st, logits, select_bias, *rule, s.T, s.E, s.k, s.renorm, topk_idx, topk_w);
    MOE_LAUNCH_CHECK("gate_select_kernel");
    return MOE_OK;
}
