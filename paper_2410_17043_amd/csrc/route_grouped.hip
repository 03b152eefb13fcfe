// Gate with scores, a balance bias and groups of experts.
//
//   l = x . Wg^T;  s = softmax(l) or sigmoid(l);  c = s + bias;  the top_groups groups of the largest rank;  the k largest c in them
//
// Logits on the matrix cores: a block takes 16 MT tokens and all experts over H or a piece of it.  Many tokens: the block selects for its
// tokens as well (one kernel, the logits never leave the CU), and so where its weights are small.  Else, with few tokens: H is cut into pieces over more
// blocks, the pieces' sums go to the workspace, and a second kernel adds and selects.  Selection: 16 lanes per token.
//
// Times: 16384 tokens of 2048, 64 experts 17.9 us (one kernel; 68 MB at 3.8 TB/s, start and selection included); 64 tokens 10 us (6.2 and 4.3: two
// chains of a launch, a round trip and a selection); 4096 tokens of 4096, 256 experts 27.8 us (19.2, of which about 7 are the start and the 16.8 MB of pieces and 0.75 a
// step of 40 KB per CU; and 10.4).
#include "common.h"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kStep = 128;                                   // bytes of a row per step; operands: 16 bytes of each half per lane (the order of the sum is free)

// ------------------------------------------------------------------------------------------------ selection
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true)); }
// over the 16 lanes of a row, in every lane: row_ror by 8, 4, 2, 1
__device__ __forceinline__ float max16(float v) {
    v = fmaxf(v, dpp<0x128>(v)); v = fmaxf(v, dpp<0x124>(v)); v = fmaxf(v, dpp<0x122>(v));
    return fmaxf(v, dpp<0x121>(v));
}
__device__ __forceinline__ float sum16(float v) {
    v += dpp<0x128>(v); v += dpp<0x124>(v); v += dpp<0x122>(v);
    return v + dpp<0x121>(v);
}
// LDS written by a wave and read back by it: its accesses execute in order, the compiler has to keep them so
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

__host__ __device__ inline int scratch_floats(int E, int n_groups) { return (E + n_groups + 16 + 3) & ~3; }   // of a token: selection scores, group ranks, the list

// The two largest of two pairs a >= b
__device__ __forceinline__ void merge2(float& a, float& b, float oa, float ob) {
    b = fmaxf(fminf(a, oa), fmaxf(b, ob));
    a = fmaxf(a, oa);
}

// Whether each lane's experts lie in one group and a group is 1, 2, 4, 8 or 16 neighbouring lanes: ranks then cross lanes without LDS
__host__ __device__ inline bool groups_of_lanes(int size, int nc) { return size % nc == 0 && size / nc <= 16 && ((size / nc) & (size / nc - 1)) == 0; }

// Drops the experts of the groups that are not kept: c = minus infinity.  scratch: LDS of this token.
template <int NC>
__device__ __forceinline__ void keep_groups(float (&c)[NC], float* scratch, const moe_gate_rule& rule, int E, int sub, int base) {
    const int size = E / rule.n_groups;
    const bool two = rule.group_rank == MOE_GROUP_TOP2 && size > 1;
    if (groups_of_lanes(size, NC)) {
        const int lanes = size / NC, mine = sub / lanes;     // (lanes beyond the last expert have groups beyond the last, of rank minus infinity)
        float a = c[0], b = -INFINITY;
#pragma unroll
        for (int i = 1; i < NC; ++i) merge2(a, b, c[i], -INFINITY);
        if (lanes > 1) merge2(a, b, dpp<0xB1>(a), dpp<0xB1>(b));       // lane ^ 1
        if (lanes > 2) merge2(a, b, dpp<0x4E>(a), dpp<0x4E>(b));       // lane ^ 2
        if (lanes > 4) merge2(a, b, dpp<0x141>(a), dpp<0x141>(b));     // the other quad of the half row (mirrored: its lanes agree)
        if (lanes > 8) merge2(a, b, dpp<0x140>(a), dpp<0x140>(b));     // the other half of the row
        float rank = two ? a + b : a;
        if (!(rank == rank)) rank = -INFINITY;
        int before = 0;
        for (int o = 0; o < rule.n_groups; ++o) {
            const float v = __shfl(rank, base + o * lanes, 64);
            before += v > rank || (v == rank && o < mine);
        }
        if (before >= rule.top_groups) {
#pragma unroll
            for (int i = 0; i < NC; ++i) c[i] = -INFINITY;
        }
        return;
    }
    float* const rank = scratch + E;
    in_order();
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (sub * NC + i < E) scratch[sub * NC + i] = c[i];
    in_order();
    for (int g = sub; g < rule.n_groups; g += 16) {
        float a = -INFINITY, b = -INFINITY;                  // the two largest
        int at = g % size;                                   // lanes start at different elements: different banks
        for (int i = 0; i < size; ++i) {
            merge2(a, b, scratch[g * size + at], -INFINITY);
            at = at + 1 == size ? 0 : at + 1;
        }
        const float r = two ? a + b : a;
        rank[g] = r == r ? r : -INFINITY;
    }
    in_order();
    uint32_t kept = 0;                                       // of this lane's groups
    for (int g = sub, n = 0; g < rule.n_groups; g += 16, ++n) {
        const float mine = rank[g];
        int before = 0;
        for (int o = 0; o < rule.n_groups; ++o) {
            const float v = rank[o];
            before += v > mine || (v == mine && o < g);
        }
        if (before < rule.top_groups) kept |= 1u << n;
    }
    in_order();
    for (int g = sub, n = 0; g < rule.n_groups; g += 16, ++n) rank[g] = kept >> n & 1 ? 1.f : 0.f;
    in_order();
    int g = sub * NC / size, at = sub * NC - g * size;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (sub * NC + i < E && rank[g] == 0.f) c[i] = -INFINITY;
        if (++at == size) { at = 0; ++g; }
    }
}

// One token by 16 lanes (sub = 0 .. 15), which look after the NC experts sub NC ...; l: its logits (minus infinity beyond E), row: the same in LDS.
// scratch: LDS of this token, scratch_floats.  bias_of: of this lane's experts.  All lanes of a wave take part (live: whether there is a token).
template <int NC>
__device__ __forceinline__ void select_token(const float (&l)[NC], const float* row, float* scratch, const float (&bias_of)[NC], const moe_gate_rule& rule, int E, int k, int renorm,
                                             int sub, bool live, int32_t* idx_out, float* w_out) {
    const int base = threadIdx.x & 48;                       // first lane of this token
    float top = 0.f, total = 1.f, c[NC];
    if (rule.score == MOE_SCORE_SOFTMAX) {
        top = l[0];
#pragma unroll
        for (int i = 1; i < NC; ++i) top = fmaxf(top, l[i]);
        top = max16(top);
        total = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) total += c[i] = expf(l[i] - top);   // a NaN makes the sum one, and with it every score
        total = sum16(total);
#pragma unroll
        for (int i = 0; i < NC; ++i) c[i] /= total;
    } else {
#pragma unroll
        for (int i = 0; i < NC; ++i) c[i] = 1.f / (1.f + expf(-l[i]));
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        c[i] += bias_of[i];
        if (sub * NC + i >= E || !(c[i] == c[i])) c[i] = -INFINITY;
    }
    if (rule.top_groups < rule.n_groups) keep_groups<NC>(c, scratch, rule, E, sub, base);
    int* const list = reinterpret_cast<int*>(scratch + E + rule.n_groups);
    in_order();
    list[sub] = -1;
    in_order();
    for (int j = 0; j < k; ++j) {
        float best = c[0];
#pragma unroll
        for (int i = 1; i < NC; ++i) best = fmaxf(best, c[i]);
        const float m = max16(best);
        // the lanes' experts ascend with the lane: the first lane that has the maximum has the lowest expert
        const uint32_t have = (uint32_t)(__ballot(best == m) >> base) & 0xffffu;
        if (sub == __builtin_ctz(have) && m > -INFINITY) {
            int at = NC - 1;
#pragma unroll
            for (int i = NC - 1; i >= 0; --i) at = c[i] == m ? i : at;
#pragma unroll
            for (int i = 0; i < NC; ++i) c[i] = i == at ? -INFINITY : c[i];
            list[j] = sub * NC + at;
        }
    }
    in_order();
    const int my_idx = list[sub];
    float w = 0.f;
    if (my_idx >= 0) {
        const float v = row[my_idx];
        w = rule.score == MOE_SCORE_SOFTMAX ? expf(v - top) / total : 1.f / (1.f + expf(-v));
    }
    if (renorm) {
        const float sum = sum16(w);                          // (lanes beyond k have none)
        w = sum > 0.f ? w / sum : 0.f;
    }
    if (live && sub < k) {
        idx_out[sub] = my_idx;
        w_out[sub] = w * rule.scale;
    }
}
template <int NC> __device__ __forceinline__ void load_bias(float (&b)[NC], const float* __restrict__ bias, int E, int sub) {
#pragma unroll
    for (int i = 0; i < NC; ++i) b[i] = bias && sub * NC + i < E ? bias[sub * NC + i] : 0.f;
}

// ------------------------------------------------------------------------------------------------ logits
struct GateArgs {
    const char *x, *wg;
    const float* bias;
    float* parts;            // [pieces][T][Ep] or unused
    int32_t* idx;
    float* w;
    int T, H, E, Ep, k, renorm;
    moe_gate_rule rule;
};

// 16 tokens per block and up to 64 experts: each of the 8 waves takes all 16 NT experts and every eighth step of H, operands in registers: the shortest chain for few steps
// (64 tokens of 2048, 64 experts in four pieces: a step per wave, 6.2 us)
template <int DT, int NT, bool FUSED>
__global__ __launch_bounds__(64 * kWaves, 2) void gate_logits_kernel(GateArgs g) {
    constexpr int D = 4, MT = 1, FRAGS = NT * MT, NC = NT;
    extern __shared__ __attribute__((aligned(16))) f32x4 part[];   // [8][FRAGS][64]; then the logits [16 MT][Ep + 4] and the scratch of the selection
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, quarter = lane >> 4;
    const int t0 = blockIdx.x * 16 * MT;
    const uint32_t pitch = (uint32_t)g.H * (DT == MOE_BF16 ? 2 : 4);
    const int steps = (int)((pitch + kStep - 1) / kStep);
    const int s0 = (int)((int64_t)steps * blockIdx.y / gridDim.y), n_all = (int)((int64_t)steps * (blockIdx.y + 1) / gridDim.y) - s0;
    const int n = (n_all - wave + kWaves - 1) / kWaves;      // steps s0 + wave, + 8, ...
    auto rsrc = [](const char* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, bytes, 0x00027000); };
    const int rows = min(16 * MT, g.T - t0), experts = min(16 * NT, g.E);
    const __amdgpu_buffer_rsrc_t xr = rsrc(g.x + (size_t)t0 * pitch, (uint32_t)rows * pitch);
    const __amdgpu_buffer_rsrc_t wr = rsrc(g.wg, (uint32_t)experts * pitch);
    uint32_t x_off[MT], w_off[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x_off[i] = (uint32_t)min(16 * i + r, rows - 1) * pitch;
#pragma unroll
    for (int j = 0; j < NT; ++j) w_off[j] = (uint32_t)min(16 * j + r, experts - 1) * pitch;
    float bias[NC];
    if (FUSED) load_bias<NC>(bias, g.bias, g.E, r);
    struct Step { u32x4 x[MT][2], w[NT][2]; };
    auto load = [&](Step& s, int i) {
        // past the end nothing is fetched (zeros from outside the row): the count of outstanding loads stays uniform
        const uint32_t at = i < n ? (uint32_t)(s0 + wave + i * kWaves) * kStep + quarter * 16 : pitch;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t in_row = at + 64 * h;
            const bool in = in_row < pitch;                  // rows are multiples of 16 bytes: a chunk is inside or not; outside the descriptor reads as zeros
#pragma unroll
            for (int q = 0; q < MT; ++q) s.x[q][h] = __builtin_amdgcn_raw_buffer_load_b128(xr, in ? x_off[q] + in_row : 0xFFFFFFF0u, 0, 0);
#pragma unroll
            for (int q = 0; q < NT; ++q) s.w[q][h] = __builtin_amdgcn_raw_buffer_load_b128(wr, in ? w_off[q] + in_row : 0xFFFFFFF0u, 0, 0);
        }
    };
    f32x4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Step& s) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (DT == MOE_BF16) {
                        acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, s.w[j][h]), __builtin_bit_cast(bf16x8, s.x[i][h]), acc[j][i], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(s.w[j][h][e]), __uint_as_float(s.x[i][h][e]), acc[j][i], 0, 0, 0);
                    }
                }
    };
    Step s[D];
#pragma unroll
    for (int d = 0; d < D; ++d) load(s[d], d);
    int i = 0;
    for (; i + D <= n; i += D)
#pragma unroll
        for (int d = 0; d < D; ++d) {
            multiply(s[d]);
            load(s[d], i + d + D);
        }
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (i + d < n) multiply(s[d]);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < MT; ++q) part[(wave * FRAGS + j * MT + q) * 64 + lane] = acc[j][q];
    __syncthreads();
    // fragment (j, q) of all experts: lane: token 16 q + lane % 16, experts 16 j + 4 (lane / 16) ...
    constexpr int PER_WAVE = (FRAGS + kWaves - 1) / kWaves;
    f32x4 sum[PER_WAVE];
#pragma unroll
    for (int u = 0; u < PER_WAVE; ++u) {
        const int f = min(u * kWaves + wave, FRAGS - 1);
        sum[u] = part[f * 64 + lane];
#pragma unroll
        for (int p = 1; p < kWaves; ++p) sum[u] += part[(p * FRAGS + f) * 64 + lane];
    }
    if (FUSED) __syncthreads();
    float* const logits = reinterpret_cast<float*>(part);
    const int row_floats = g.Ep + 4;
#pragma unroll
    for (int u = 0; u < PER_WAVE; ++u) {
        const int f = u * kWaves + wave, token = 16 * (f % MT) + r, e = 16 * (f / MT) + 4 * quarter;
        if (f >= FRAGS || e >= g.Ep) continue;
        if (FUSED) *reinterpret_cast<f32x4*>(logits + token * row_floats + e) = sum[u];
        else if (t0 + token < g.T) *reinterpret_cast<f32x4*>(g.parts + ((size_t)blockIdx.y * g.T + t0 + token) * g.Ep + e) = sum[u];
    }
    if (!FUSED) return;
    __syncthreads();
    float* const scratch = logits + 16 * MT * row_floats + (wave * 4 + quarter) * scratch_floats(g.E, g.rule.n_groups);
    for (int token = wave * 4 + quarter; token < 16 * MT; token += 4 * kWaves) {   // the same number of turns for all waves: 16 MT is a multiple or MT = 1
        float l[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) l[c] = r * NC + c < g.E ? logits[token * row_floats + r * NC + c] : -INFINITY;
        const int t = t0 + token;
        select_token<NC>(l, logits + token * row_floats, scratch, bias, g.rule, g.E, g.k, g.renorm, r, t < g.T, g.idx + (size_t)t * g.k, g.w + (size_t)t * g.k);
    }
}

// 64 tokens per block, or more than 64 experts: each of the 8 waves takes a part of the tokens and 16 NT experts over the whole piece of H.  Weights and tokens go through a ring of D + 1 steps
// in LDS, 8 rows of a whole 128-byte line per load.  One barrier per step.  4096 tokens of 4096, 256 experts: 19.2 us (three steps ahead 19.5); with the weights in registers, loads of 16
// rows of half a line, 23.4; waves that each fetch their tokens too 41.  16384 tokens of 2048, 64 experts, with the selection: 17.9 us (seven steps ahead 19.0); waves that share H out instead and add
// their sums through LDS, all operands in registers, 25.9; 32 experts 16.3 and 20.3, 8 experts of 4096 34.2 and 34.1.
__device__ __forceinline__ int token_swizzle(int row) { return (row >> 1) & 7; }
// WT: the waves are WT parts of the tokens times kWaves / WT parts of the experts
template <int MT, int NT, int WT> struct WideGeom {
    static constexpr int WE = kWaves / WT, D = WT > 1 ? 3 : 2;           // steps ahead
    static constexpr int TOKENS = 16 * MT * kStep, OWN = 16 * NT * kStep, STAGE = TOKENS + WE * OWN, LDS = (D + 1) * STAGE;
};
template <int DT, int MT, int NT, int WT, bool FUSED>
__global__ __launch_bounds__(64 * kWaves, 2) void gate_logits_wide_kernel(GateArgs g) {
    using WG = WideGeom<MT, NT, WT>;
    constexpr int D = WG::D, TOKENS = WG::TOKENS, OWN = WG::OWN, STAGE = WG::STAGE, LOADERS = 2 * MT, NC = WG::WE * NT, MQ = MT / WT, WL = 2 * NT > WT ? 2 * NT / WT : 1;
    static_assert(MT % WT == 0, "");
    extern __shared__ __attribute__((aligned(1024))) unsigned char ring[];   // D + 1 stages; then the logits [16 MT][Ep + 4] and the scratch of the selection
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, quarter = lane >> 4;
    const int t0 = blockIdx.x * 16 * MT, part = wave % WG::WE, tokens0 = wave / WG::WE * MQ, e0 = part * 16 * NT;   // tokens0: in 16
    const uint32_t pitch = (uint32_t)g.H * (DT == MOE_BF16 ? 2 : 4);
    const int steps = (int)((pitch + kStep - 1) / kStep);
    const int s0 = (int)((int64_t)steps * blockIdx.y / gridDim.y), n = (int)((int64_t)steps * (blockIdx.y + 1) / gridDim.y) - s0;   // n >= 1 (see plan_gate)
    auto rsrc = [](const char* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, bytes, 0x00027000); };
    const int rows = min(16 * MT, g.T - t0), experts = max(1, min(16 * NT, g.E - e0));
    const __amdgpu_buffer_rsrc_t xr = rsrc(g.x + (size_t)t0 * pitch, (uint32_t)rows * pitch);
    const __amdgpu_buffer_rsrc_t wr = rsrc(g.wg + (size_t)min(e0, g.E - 1) * pitch, (uint32_t)experts * pitch);
    // 8 rows of a stage per wave-load; with fewer than 64 tokens several waves fetch the same ones (to the same place)
    const int loader = wave % LOADERS, my_row = 8 * loader + (lane >> 3);
    const uint32_t x_off = (uint32_t)min(my_row, rows - 1) * pitch, x_chunk = ((lane & 7) ^ token_swizzle(my_row & 15)) << 4;
    float bias[NC];
    if (FUSED) load_bias<NC>(bias, g.bias, g.E, r);
    auto at_step = [&](int i) { return i < n ? (uint32_t)(s0 + i) * kStep : pitch; };   // past the end nothing is fetched (zeros from outside the row): the count of outstanding loads stays uniform
    auto load_tokens = [&](int i, int stage) {
        const uint32_t in_row = at_step(i) + x_chunk;        // rows are multiples of 16 bytes; outside the descriptor reads as zeros
        load_to_lds(xr, ring + stage * STAGE + loader * 1024, in_row < pitch ? x_off + in_row : 0xFFFFFFF0u, 0);
    };
    uint32_t w_off[WL];
    const int w_first = wave / WG::WE * WL % (2 * NT), w_row = 8 * w_first + (lane >> 3);
#pragma unroll
    for (int u = 0; u < WL; ++u) w_off[u] = (uint32_t)min(w_row + 8 * u, experts - 1) * pitch;
    auto load_weights = [&](int i, int stage) {
#pragma unroll
        for (int u = 0; u < WL; ++u) {
            const uint32_t in_row = at_step(i) + (((lane & 7) ^ token_swizzle((w_row + 8 * u) & 15)) << 4);
            load_to_lds(wr, ring + stage * STAGE + TOKENS + part * OWN + (w_first + u) * 1024, in_row < pitch ? w_off[u] + in_row : 0xFFFFFFF0u, 0);
        }
    };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_tokens(d, d);
        load_weights(d, d);
    }
    f32x4 acc[NT][MQ];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MQ; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int frag = r * kStep + ((quarter ^ token_swizzle(r)) << 4);
    int stage = 0;
    for (int i = 0; i < n; ++i) {
        // what was issued for steps i + 1 .. i + D - 1 may be outstanding; lgkmcnt(0): this wave has read the stage that is refilled below
        constexpr int OPEN = (D - 1) * (WL + 1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (OPEN & 15) | (OPEN >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        load_tokens(i + D, stage == 0 ? D : stage - 1);
        load_weights(i + D, stage == 0 ? D : stage - 1);
        const unsigned char *const st = ring + stage * STAGE, *const own = st + TOKENS + part * OWN;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 w[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) w[j] = *reinterpret_cast<const u32x4*>(own + (frag ^ (64 * h)) + j * 16 * kStep);
#pragma unroll
            for (int q = 0; q < MQ; ++q) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(st + (frag ^ (64 * h)) + (tokens0 + q) * 16 * kStep);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (DT == MOE_BF16) {
                        acc[j][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[j]), __builtin_bit_cast(bf16x8, x), acc[j][q], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][q] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j][e]), __uint_as_float(x[e]), acc[j][q], 0, 0, 0);
                    }
                }
            }
        }
        stage = stage == D ? 0 : stage + 1;
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                      // no load may still target LDS
    float* const logits = reinterpret_cast<float*>(ring);
    const int row_floats = g.Ep + 4;
    if (FUSED) __syncthreads();
    // lane: token 16 q + lane % 16, experts e0 + 16 j + 4 (lane / 16) ...
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < MQ; ++q) {
            const int token = 16 * (tokens0 + q) + r, e = e0 + 16 * j + 4 * quarter;
            if (e >= g.Ep) continue;
            if (FUSED) *reinterpret_cast<f32x4*>(logits + token * row_floats + e) = acc[j][q];
            else if (t0 + token < g.T) *reinterpret_cast<f32x4*>(g.parts + ((size_t)blockIdx.y * g.T + t0 + token) * g.Ep + e) = acc[j][q];
        }
    if (!FUSED) return;
    __syncthreads();
    float* const scratch = logits + 16 * MT * row_floats + (wave * 4 + quarter) * scratch_floats(g.E, g.rule.n_groups);
    for (int token = wave * 4 + quarter; token < 16 * MT; token += 4 * kWaves) {
        float l[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) l[c] = r * NC + c < g.E ? logits[token * row_floats + r * NC + c] : -INFINITY;
        const int t = t0 + token;
        select_token<NC>(l, logits + token * row_floats, scratch, bias, g.rule, g.E, g.k, g.renorm, r, t < g.T, g.idx + (size_t)t * g.k, g.w + (size_t)t * g.k);
    }
}

// Adds the pieces of H and selects; 16 tokens per block.  Lanes fetch 16 neighbouring bytes each, 256 per token, and take their own experts from LDS.
template <int NC>
__global__ __launch_bounds__(256) void gate_select_kernel(GateArgs g, int pieces) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int lane = threadIdx.x & 63, sub = lane & 15, slot = (threadIdx.x >> 6) * 4 + (lane >> 4);
    const int t = blockIdx.x * 16 + slot;
    const bool live = t < g.T;
    const float* const from = g.parts + (size_t)min(t, g.T - 1) * g.Ep;
    constexpr int Q = (NC + 3) / 4;                          // 16-byte units per lane
    float* const row = lds + g.Ep + slot * (g.Ep + scratch_floats(g.E, g.rule.n_groups));
    f32x4 sum[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float my_bias = g.bias && (int)threadIdx.x < g.E ? g.bias[threadIdx.x] : 0.f;
    for (int p0 = 0; p0 < pieces; p0 += 4) {                 // four pieces are requested before the first is added (past the last one that again, not added)
        f32x4 v[4][Q];
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < Q; ++q)
                v[p][q] = *reinterpret_cast<const f32x4*>(from + (size_t)min(p0 + p, pieces - 1) * g.T * g.Ep + min(4 * (sub + 16 * q), g.Ep - 4));
#pragma unroll
        for (int p = 0; p < 4; ++p)
            if (p0 + p < pieces)
#pragma unroll
                for (int q = 0; q < Q; ++q) sum[q] += v[p][q];
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (4 * (sub + 16 * q) < g.Ep) *reinterpret_cast<f32x4*>(row + 4 * (sub + 16 * q)) = sum[q];
    if ((int)threadIdx.x < g.E) lds[threadIdx.x] = my_bias;
    __syncthreads();
    float l[NC], bias[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e = sub * NC + c;
        l[c] = e < g.E ? row[e] : -INFINITY;
        bias[c] = e < g.E ? lds[e] : 0.f;
    }
    select_token<NC>(l, row, row + g.Ep, bias, g.rule, g.E, g.k, g.renorm, sub, live, g.idx + (size_t)t * g.k, g.w + (size_t)t * g.k);
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int padded_experts(int E) { return (E + 3) & ~3; }

// How a gate is run: tokens per block / 16, pieces of H (0: one kernel)
struct GatePlan { int mt, pieces; };
constexpr int kGateCUs = 256;
// One kernel of 16 tokens per block where a block's tokens and weights are this few bytes, and the blocks a round or their selection short: 16 experts of 1024, 512 tokens
// 7.3 -> 6.0 us, 4096 9.8 -> 6.3; 64 of 512 9.6 -> 8.1 and 11.8 -> 8.6, but 11000 tokens 13.3 -> 22.8.  Of more bytes two kernels are faster: 8 experts of 4096 (192 KB) 7.5 and 10.0
constexpr size_t kSmallGate = 96 * 1024;
GatePlan plan_gate(const moe_shape& s) {
    const int steps = (int)(((int64_t)s.H * elem_size(s.dtype) + kStep - 1) / kStep);
    const int least = s.E <= 64 ? kWaves : 4;                // steps per piece, at least
    GatePlan p;
    p.mt = s.T >= 1024 ? 4 : 1;
    const int blocks = (s.T + 16 * p.mt - 1) / (16 * p.mt);
    p.pieces = blocks * 4 >= 3 * kGateCUs ? 0 : std::max(1, std::min(kGateCUs / blocks, steps / least));
    if (p.pieces == 0) p.mt = 4;
    else if (s.E <= 64 && (size_t)(16 + s.E) * s.H * elem_size(s.dtype) <= kSmallGate && ((s.T + 15) / 16 <= kGateCUs || s.E <= 16)) p = GatePlan{1, 0};
    return p;
}

// WT: 0: gate_logits_kernel
template <int MT, int NT, int WT> constexpr int most_experts() { return 16 * NT * (WT > 0 ? kWaves / WT : 1); }   // that the instantiation takes
template <int MT, int NT, int WT, bool FUSED> int logits_lds(int E, int n_groups) {
    const int bytes = WT > 0 ? WideGeom<MT, NT, WT ? WT : 1>::LDS : kWaves * NT * MT * 1024;
    return FUSED ? std::max(bytes, (16 * MT * (padded_experts(E) + 4) + 4 * kWaves * scratch_floats(E, n_groups)) * 4) : bytes;
}
struct GateLds { int bytes, limit; };                        // of a launch; what its kernel's limit is set to, whatever the launch
template <int DT, int MT, int NT, int WT, bool FUSED>
int launch_logits(const GateArgs& g, int pieces, hipStream_t st, GateLds* only_lds) {
    constexpr int E = most_experts<MT, NT, WT>();
    const GateLds lds = {logits_lds<MT, NT, WT, FUSED>(g.E, g.rule.n_groups), logits_lds<MT, NT, WT, FUSED>(E, E)};
    if (only_lds) { *only_lds = lds; return MOE_OK; }
    void (*kernel)(GateArgs);
    if constexpr (WT > 0) kernel = &gate_logits_wide_kernel<DT, MT, NT, WT, FUSED>;
    else kernel = &gate_logits_kernel<DT, NT, FUSED>;
    // to the most that any launch needs
    static LdsLimit limit;
    if (const int rc = raise_lds_limit(limit, reinterpret_cast<const void*>(kernel), lds.limit)) return rc;
    hipLaunchKernelGGL(kernel, dim3((g.T + 16 * MT - 1) / (16 * MT), FUSED ? 1 : pieces), dim3(64 * kWaves), lds.bytes, st, g);
    MOE_LAUNCH_CHECK("gate_logits_kernel");
    return MOE_OK;
}
template <int DT, int MT, bool FUSED>
int launch_logits_e(const GateArgs& g, int pieces, hipStream_t st, GateLds* only_lds = nullptr) {
    if constexpr (MT == 4) {
        if (g.E <= 32) return launch_logits<DT, MT, 1, 4, FUSED>(g, pieces, st, only_lds);
        if (g.E <= 64) return launch_logits<DT, MT, 1, 2, FUSED>(g, pieces, st, only_lds);
    } else {
        if (g.E <= 16) return launch_logits<DT, MT, 1, 0, FUSED>(g, pieces, st, only_lds);
        if (g.E <= 32) return launch_logits<DT, MT, 2, 0, FUSED>(g, pieces, st, only_lds);
        if (g.E <= 64) return launch_logits<DT, MT, 4, 0, FUSED>(g, pieces, st, only_lds);
    }
    if constexpr (MT == 1 && FUSED) return moe_set_error(MOE_EINTERNAL, "no gate of 16 tokens per block selects from %d experts", g.E);   // see plan_gate
    else return g.E <= 128 ? launch_logits<DT, MT, 1, 1, FUSED>(g, pieces, st, only_lds) : launch_logits<DT, MT, 2, 1, FUSED>(g, pieces, st, only_lds);
}
// Tokens per launch of the one kernel, at 8 or 32 threads each: of 2^32 threads and more only the number modulo 2^32 would run, with no error
constexpr int kLaunchTokens = 1 << 26;
template <int DT>
int launch_gate(const GateArgs& all, const GatePlan& p, hipStream_t st) {
    GateArgs g = all;
    if (p.pieces == 0) {
        for (int64_t t = 0; t < all.T; t += kLaunchTokens) {
            g.T = (int)std::min<int64_t>(kLaunchTokens, all.T - t);
            g.x = all.x + t * g.H * (DT == MOE_BF16 ? 2 : 4);
            g.idx = all.idx + t * g.k;
            g.w = all.w + t * g.k;
            const int rc = p.mt == 4 ? launch_logits_e<DT, 4, true>(g, 0, st) : launch_logits_e<DT, 1, true>(g, 0, st);
            if (rc != MOE_OK) return rc;
        }
        return MOE_OK;
    }
    const int rc = p.mt == 4 ? launch_logits_e<DT, 4, false>(g, p.pieces, st) : launch_logits_e<DT, 1, false>(g, p.pieces, st);
    if (rc != MOE_OK) return rc;
    const int bytes = (g.Ep + 16 * (g.Ep + scratch_floats(g.E, g.rule.n_groups))) * 4;   // at most 50 KB
#define MOE_SELECT(NC) hipLaunchKernelGGL(gate_select_kernel<NC>, dim3((g.T + 15) / 16), dim3(256), bytes, st, g, p.pieces)
    if (g.E <= 16) MOE_SELECT(1);
    else if (g.E <= 32) MOE_SELECT(2);
    else if (g.E <= 64) MOE_SELECT(4);
    else if (g.E <= 128) MOE_SELECT(8);
    else MOE_SELECT(16);
#undef MOE_SELECT
    MOE_LAUNCH_CHECK("gate_select_kernel");
    return MOE_OK;
}

}  // namespace

extern "C" int moe_selfcheck_gate_plan(int32_t T, int32_t H, int32_t E, int32_t n_groups, int32_t dtype, int32_t* plan4) {
    const moe_shape s = {T, H, E, 1, 1, dtype, 0, 0};
    const int rc = moe_check_shape(&s);
    if (rc != MOE_OK) return rc;
    if (n_groups < 1 || E % n_groups != 0 || !plan4) return moe_set_error(MOE_EINVAL, "moe_selfcheck_gate_plan: bad argument");
    const GatePlan p = plan_gate(s);
    GateArgs g = {};
    g.T = T; g.H = H; g.E = E; g.Ep = padded_experts(E);
    g.rule.n_groups = n_groups;
    GateLds lds = {0, 0};
    if (p.pieces == 0) p.mt == 4 ? launch_logits_e<MOE_F32, 4, true>(g, 0, nullptr, &lds) : launch_logits_e<MOE_F32, 1, true>(g, 0, nullptr, &lds);
    else p.mt == 4 ? launch_logits_e<MOE_F32, 4, false>(g, p.pieces, nullptr, &lds) : launch_logits_e<MOE_F32, 1, false>(g, p.pieces, nullptr, &lds);
    plan4[0] = 16 * p.mt; plan4[1] = p.pieces; plan4[2] = lds.bytes; plan4[3] = lds.limit;
    const int steps = (int)(((int64_t)H * elem_size(dtype) + kStep - 1) / kStep);
    if (p.pieces > steps) return moe_set_error(MOE_EINTERNAL, "a piece without steps");
    if (lds.bytes <= 0 || lds.bytes > lds.limit || lds.limit > 160 * 1024) return moe_set_error(MOE_EINTERNAL, "LDS: %d bytes, limit %d", lds.bytes, lds.limit);
    return MOE_OK;
}

extern "C" size_t moe_route_grouped_workspace_bytes(const moe_ctx* ctx) {
    if (!ctx) return 0;
    return align256(std::max<size_t>((size_t)plan_gate(ctx->s).pieces * ctx->s.T * padded_experts(ctx->s.E) * sizeof(float), 1));
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
    if ((int64_t)s.H * elem_size(s.dtype) > 1 << 24) return moe_set_error(MOE_ESHAPE, "moe_route_grouped: rows of at most 16 MiB");
    if (!aligned16(x) || !aligned16(Wg) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return moe_set_error(MOE_EALIGN, "moe_route_grouped: x, Wg need 16-byte, workspace 256-byte alignment");
    if (workspace_bytes < moe_route_grouped_workspace_bytes(ctx))
        return moe_set_error(MOE_ESHAPE, "moe_route_grouped: workspace too small (%zu < %zu)", workspace_bytes, moe_route_grouped_workspace_bytes(ctx));
    ctx->rank_src = nullptr;                                 // new indices: no ranks to reuse
    const GateArgs g = {reinterpret_cast<const char*>(x), reinterpret_cast<const char*>(Wg), select_bias, reinterpret_cast<float*>(workspace), topk_idx, topk_w,
                        s.T, s.H, s.E, padded_experts(s.E), s.k, s.renorm, *rule};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return s.dtype == MOE_BF16 ? launch_gate<MOE_BF16>(g, plan_gate(s), st) : launch_gate<MOE_F32>(g, plan_gate(s), st);
}
