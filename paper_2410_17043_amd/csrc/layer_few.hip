// A whole layer for a few tokens: gate, then two kernels that stream the weights of the experts that some token chose.
//
//   up:    h[t,e] = act(W1_e x_t [, Wu_e x_t])           a block per 16 inner columns of an expert, for the tokens that chose it
//   down:  y[t] = sum_j w[t,j] Wd_e h[t,e] (+ shared)    a block per 16 columns and expert; the last one of the columns adds the experts up in the tokens' order
//
// Bound by memory: every weight of a chosen expert is read once, straight to registers, 128 bytes of each row a step, which the block's waves share out; the tokens, up
// to 64, are the other side of the matrix instructions.  No send buffer, no segments: the kernels find the experts in the list of choices, and a product's rows are the
// tokens' own.
//
// Sums in fp32.  h is kept as two bf16 numbers (its rounding, and the rounding of what is left: 2^-17) in bf16 layers, as the matrix cores have time for both beside the
// weights' way in, so that y, rounded once, is what the products give: 0.0017 of its norm off 64 bits instead of 0.0024.  No atomic adds: results do not change from run to run.
#include "ffn_tiles.h"
#include "lanes.h"
#include <type_traits>

namespace {

// A lane each.  By route, dispatch, expert FFN and combine instead (whole layers in a graph, weights beyond the caches, 1, 8, 16, 32 and 64 tokens): bf16, 2048 -> 1408 SwiGLU, six of 64
// experts 52, 171, 216, 245, 249 us, by these kernels 46, 160, 215, 259, 332; 4096 -> 14336 SwiGLU, two of eight 173, 471, 508, 518, 536 and 159, 453, 537, 603, 738; 1024 -> 4096 GELU,
// one of 16 29, 47, 63, 76, 84 and 22, 41, 53, 76, 92; fp32, 1024 -> 4096 SwiGLU, two of eight, 1, 16, 64 tokens 107, 194, 197 and 45, 101, 124.
constexpr int kFewTokens = 64;
constexpr int kFewWidth = 1 << 18;                           // of H and F: offsets of 32 bits
constexpr int kFewWaves = 4, kChunk = 128;                   // bytes of a row that a wave takes at a time

struct FewArgs {
    ExpertTable tab;                 // of the experts here
    int8_t local[MOE_MAX_E];         // place in the table of every expert of the layer, -1: on another GPU
    const void *s1, *s_up, *s_down;  // the shared expert
    const void* x;
    int32_t* idx;
    float* w;
    const void* gate;                // [E, H]
    const float* gate_bias;
    double* logits;                  // [T, E]
    int32_t* gate_done;              // per tile of tokens
    void *h, *h_shared;              // [T k, F], [T, F_shared]; in bf16 layers what their roundings leave behind each
    float* parts;                    // [T k + T, H]: weighted sums of every choice, of the shared expert
    int32_t* done;                   // [ceil(H / 16)]: experts that have arrived, per tile of columns
    void* y;
    int T, H, F, F_shared, E, k, renorm;
    int shared_here;                 // whether the launch does the shared expert's tiles
    int clear;                       // whether it clears `done`
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t all_of(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffffu, 0x00027000); }

// The choices of a token by a wave, lane j the j-th: the k largest logits, of equal ones the lower expert first, and their weights
struct Choice { int expert; float weight; };
template <class Logit> __device__ __forceinline__ Choice select(const FewArgs& a, Logit logit) {
    const int lane = threadIdx.x & 63;
    // the lane's logits, of experts lane + 64 i: as whole numbers in their order (zeros alike, NaN last), 0 once taken or not there
    double z[4];
    uint64_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        z[i] = logit(lane + 64 * i);                         // (of those that are not there: any number)
    }
    uint64_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t u = __builtin_bit_cast(uint64_t, z[i] + 0.0);
        key[i] = lane + 64 * i >= a.E ? 0 : z[i] != z[i] ? 1 : u >> 63 ? ~u : u | 1ull << 63;
        most = max(most, key[i]);
    }
    auto rotated = [](uint64_t m, auto ctrl) { return max(m, __builtin_bit_cast(uint64_t, ror<decltype(ctrl)::value>(__builtin_bit_cast(double, m)))); };
    auto of_lane = [](uint64_t m, int l) { return __builtin_bit_cast(uint64_t, lane_of(__builtin_bit_cast(double, m), l)); };
    double top = 0.0, my_z = 0.0;
    int my_e = 0;
    for (int j = 0; j < a.k; ++j) {
        uint64_t m = rotated(rotated(rotated(rotated(most, std::integral_constant<int, 0x128>{}), std::integral_constant<int, 0x124>{}), std::integral_constant<int, 0x122>{}),
                             std::integral_constant<int, 0x121>{});
        m = max(max(of_lane(m, 0), of_lane(m, 16)), max(of_lane(m, 32), of_lane(m, 48)));
        int e = -1;
        double ze = 0.0;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            const unsigned long long with = __ballot(key[i] == m);
            if (with) { e = __builtin_ctzll(with) + 64 * i; ze = lane_of(z[i], __builtin_ctzll(with)); }
        }
        if (j == 0) top = ze;
        if (lane == j) { my_z = ze; my_e = e; }
        most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (e == lane + 64 * i) key[i] = 0;
            most = max(most, key[i]);
        }
    }
    const double p = exp(my_z - top);
    double all = 0.0;
    if (a.renorm) {
        all = wave_sum(lane < a.k ? p : 0.0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.E) all += exp(z[i] - top);
        all = wave_sum(all);
    }
    return Choice{my_e, (float)(p / all)};
}

// The choices of the call: which experts of the table are used, and the table's place of each choice (-1: none here); the tables, which dynamic indexes would fetch from the
// kernel's arguments, in host memory, one round trip after the other
struct Choices {
    unsigned long long used;
    uint32_t local[MOE_MAX_E / 4];
    const void* weights[3][MOE_MAX_LOCAL];
    int8_t at[kFewTokens * MOE_MAX_K];
    float by[kFewTokens * MOE_MAX_K];                        // weights of the choices
    __device__ __forceinline__ int place(int e) const { return reinterpret_cast<const int8_t*>(local)[e]; }
};
__device__ __forceinline__ void read_choices(const FewArgs& a, Choices& c) {
    constexpr int THREADS = 64 * kFewWaves;
    static_assert(THREADS >= MOE_MAX_E / 4 && THREADS >= MOE_MAX_LOCAL, "");
    const int n = a.T * a.k, tid = threadIdx.x;
    const int first = tid < n ? a.idx[tid] : -1;             // all that is fetched goes out together
    const float weight = tid < n ? a.w[tid] : 0.f;
    if (tid < MOE_MAX_E / 4) c.local[tid] = reinterpret_cast<const uint32_t*>(a.local)[tid];
    if (tid < MOE_MAX_LOCAL) {
        c.weights[0][tid] = a.tab.w1[tid];
        c.weights[1][tid] = a.tab.w_up[tid];
        c.weights[2][tid] = a.tab.w_down[tid];
    }
    if (tid == 0) c.used = 0;
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
        const int e = i == tid ? first : a.idx[i];
        const int at = (unsigned)e < (unsigned)a.E ? c.place(e) : -1;
        c.at[i] = (int8_t)at;
        c.by[i] = i == tid ? weight : a.w[i];
        if (at >= 0) atomicOr(&c.used, 1ull << at);
    }
    __syncthreads();
}
// The tokens of an expert: lane l's place in it
struct Tokens {
    int count;                       // of the wave
    int token, row;                  // of the lane: its token and that token's first choice of the expert, as t k + j (past the count: 0)
};
__device__ __forceinline__ Tokens tokens_of(const FewArgs& a, const Choices& c, int expert) {
    const int lane = threadIdx.x & 63;
    int first = -1;
    if (lane < a.T)
        for (int j = a.k - 1; j >= 0; --j)
            if (c.at[lane * a.k + j] == expert) first = j;
    const unsigned long long has = __ballot(first >= 0);
    Tokens t;
    t.count = __builtin_popcountll(has);
    const int rank = __builtin_popcountll(has & ((1ull << lane) - 1ull)), rest = __builtin_popcountll(~has & ((1ull << lane) - 1ull));
    const int to = (first >= 0 ? rank : t.count + rest) * 4;                  // those without go behind: every lane is sent to once
    t.token = __builtin_amdgcn_ds_permute(to, first >= 0 ? lane : 0);
    t.row = __builtin_amdgcn_ds_permute(to, first >= 0 ? lane * a.k + first : 0);
    return t;
}
__device__ __forceinline__ int nth_expert(unsigned long long used, int n) {
    for (int i = 0; i < n; ++i) used &= used - 1;
    return __builtin_ctzll(used);
}
__device__ __forceinline__ const char* scalar(const void* p) {
    const uint2 u = __builtin_bit_cast(uint2, p);
    return __builtin_bit_cast(const char*, make_uint2(__builtin_amdgcn_readfirstlane(u.x), __builtin_amdgcn_readfirstlane(u.y)));
}

template <int DT> __device__ __forceinline__ void multiply(const u32x4 (&w)[2], const u32x4 (&x)[2], f32x4& acc) {
    if (DT == MOE_BF16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[i]), __builtin_bit_cast(bf16x8, x[i]), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][j]), __uint_as_float(x[i][j]), acc, 0, 0, 0);
    }
}

// 16 rows of NF weight matrices (from w[f] on, `bytes` each, the last row that there is again behind it) times 16 NT rows of `rows` (lane: row lane % 16 of tile n
// from row_off[n] on): this wave's part of the sums.  Lane: 32 bytes of a row's 128 at lane / 16; the order of a sum is free.
template <int DT, int NF, int NT, int DEPTH>
__device__ __forceinline__ void wave_sums(const char* const (&w)[NF], int last_row, uint32_t bytes, __amdgpu_buffer_rsrc_t rows, const uint32_t (&row_off)[NT], f32x4 (&acc)[NF][NT]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t part = (lane >> 4) * 32;
    const uint32_t w_off = (uint32_t)min(lane & 15, last_row) * bytes + part;
    const int chunks = (int)((bytes + kChunk - 1) / kChunk), n = (chunks - wave + kFewWaves - 1) / kFewWaves;
    if (n <= 0) return;
    u32x4 wb[DEPTH][NF][2], xb[DEPTH][NT][2];
    int at = 0;                                              // of the wave's chunks
    auto load = [&](u32x4 (&wq)[NF][2], u32x4 (&xq)[NT][2]) {
        const int byte = (at * kFewWaves + wave) * kChunk;
        ++at;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // fp32 rows may end inside the 128 bytes
            const bool in = DT == MOE_BF16 || byte + part + 16 * h < bytes;
#pragma unroll
            for (int f = 0; f < NF; ++f) wq[f][h] = __builtin_amdgcn_raw_buffer_load_b128(all_of(w[f]), in ? w_off + 16 * h : 0x80000000u, byte, 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) xq[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rows, in ? row_off[t] + part + 16 * h : 0x80000000u, byte, 0);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < n) load(wb[d], xb[d]);
    for (int i = 0; i < n; i += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (i + d < n)
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int t = 0; t < NT; ++t) multiply<DT>(wb[d][f], xb[d][t], acc[f][t]);
            if (i + d + DEPTH < n) load(wb[d], xb[d]);
        }
}

// The same, added up over the block's waves: thread i of tile t holds weight row 4 (i / 64) + i % 4 and row (i / 4) % 16 of `rows`.  PAIRS: rows 8 and on are what the roundings of
// rows 0 to 7 leave; the sums of both are in the threads of the latter.
template <int DT, int NF, int NT, bool PAIRS>
__device__ __forceinline__ void block_sums(const char* const (&w)[NF], int last_row, uint32_t bytes, __amdgpu_buffer_rsrc_t rows, const uint32_t (&row_off)[NT], float* lds, float (&out)[NF][NT]) {
    constexpr int DEPTH = NF + NT <= 2 ? 6 : NF + NT <= 3 ? 4 : NF + NT <= 4 ? 3 : NF + NT <= 5 ? 2 : 1;   // registers of four blocks on a CU
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    f32x4 acc[NF][NT];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    wave_sums<DT, NF, NT, DEPTH>(w, last_row, bytes, rows, row_off, acc);
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(lds + (((f * NT + t) * kFewWaves + wave) * 64 + lane) * 4) = acc[f][t];
    __syncthreads();
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float* const from = lds + (f * NT + t) * kFewWaves * 256;
            float v = 0.f, u = 0.f;
#pragma unroll
            for (int q = 0; q < kFewWaves; ++q) {
                v += from[q * 256 + threadIdx.x];
                if (PAIRS) u += from[q * 256 + (threadIdx.x ^ 32)];   // the lane eight further
            }
            out[f][t] = v + u;
        }
}

// One tile of 16 inner columns of an expert, or of the shared one, for its tokens.  MANY: there may be more than 16 of them.
// bf16, SwiGLU: 16 tokens of two of eight experts of 4096 x 14336 318 us (1.88 GB, 5.9 TB/s); one token of six of 64 of 2048 x 1408 and a shared expert of 2816, which the gate's launch
// has brought, 19 us (69 MB).  With every tile's chunks beginning elsewhere in its rows the former took 383 us.
template <int DT, int EPI, bool MANY>
__device__ __forceinline__ void up_tile(const FewArgs& a, const char* w1, const char* w_up, bool shared, int tile, const Tokens& tok, float* lds) {
    constexpr int NF = EPI == EPI_SWIGLU ? 2 : 1, B = DT == MOE_BF16 ? 2 : 4;
    const int width = shared ? a.F_shared : a.F, lane = threadIdx.x & 63;
    const uint32_t bytes = (uint32_t)a.H * B;
    const size_t first = (size_t)tile * 16 * bytes;
    const char* w[NF];
    w[0] = w1 + first;
    if (NF == 2) w[NF - 1] = w_up + first;
    const int last = min(15, width - 1 - tile * 16);
    char* const h = reinterpret_cast<char*>(shared ? a.h_shared : a.h);
    const size_t rest = (size_t)(shared ? a.T : a.T * a.k) * width;
    auto run = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        uint32_t row_off[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) row_off[t] = (uint32_t)__shfl(tok.token, min(16 * t + (lane & 15), tok.count - 1), 64) * bytes;
        float v[NF][NT];
        block_sums<DT, NF, NT, false>(w, last, bytes, all_of(a.x), row_off, lds, v);
        const int i = threadIdx.x, row = 4 * (i >> 6) + (i & 3);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int place = 16 * t + ((i >> 2) & 15), to = __shfl(tok.row, place, 64);
            if (place >= tok.count || row > last) continue;
            const float f = activation_fast<EPI>(v[0][t], v[NF - 1][t]);
            const size_t at = (size_t)to * width + tile * 16 + row;
            if (DT == MOE_BF16) {
                // a finite f beyond bf16's largest number keeps that one, and its rest behind it; nothing is behind an infinity (nor a NaN)
                const bool finite = fabsf(f) < __builtin_huge_valf();
                const uint32_t most = finite ? 0x7f7fu : 0x7fffu, q = f32_to_bf16_bits(f), hi = (q & 0x8000u) | min(q & 0x7fffu, most);
                const float lo = f - bf16_bits_to_f32(hi);
                reinterpret_cast<uint16_t*>(h)[at] = (uint16_t)hi;
                reinterpret_cast<uint16_t*>(h)[rest + at] = (uint16_t)(finite ? f32_to_bf16_bits(lo) : 0u);
            } else {
                reinterpret_cast<float*>(h)[at] = f;
            }
        }
    };
    if (!MANY || tok.count <= 16) return run(std::integral_constant<int, 1>{});
    if constexpr (MANY) {
        if (tok.count <= 32) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 4>{});
    }
}
__device__ __forceinline__ Tokens all_tokens(const FewArgs& a) {
    const int lane = threadIdx.x & 63, t = lane < a.T ? lane : 0;
    return Tokens{a.T, t, t};
}
template <int DT, int EPI, bool MANY> __device__ __forceinline__ void shared_tile(const FewArgs& a, int tile, float* lds) {
    up_tile<DT, EPI, MANY>(a, reinterpret_cast<const char*>(a.s1), reinterpret_cast<const char*>(a.s_up), true, tile, all_tokens(a), lds);
}
__device__ __forceinline__ void clear_done(const FewArgs& a) {
    if (a.clear && blockIdx.x == 0)
        for (int i = threadIdx.x; i < (a.H + 15) / 16; i += 64 * kFewWaves) a.done[i] = 0;
}
template <int EPI, bool MANY> constexpr int kUpLds = (EPI == EPI_SWIGLU ? 2 : 1) * (MANY ? 4 : 1) * kFewWaves * 256;

template <int DT, int EPI, bool MANY>
__global__ __launch_bounds__(64 * kFewWaves, 4) void few_up_kernel(const FewArgs a) {
    __shared__ Choices choices;
    __shared__ float lds[kUpLds<EPI, MANY>];
    clear_done(a);
    const int shared_tiles = a.shared_here ? (a.F_shared + 15) / 16 : 0, tiles = (a.F + 15) / 16;
    if ((int)blockIdx.x < shared_tiles) return shared_tile<DT, EPI, MANY>(a, blockIdx.x, lds);
    read_choices(a, choices);
    const int unit = blockIdx.x - shared_tiles, n = unit / tiles;
    if (n >= __builtin_popcountll(choices.used)) return;
    const int expert = __builtin_amdgcn_readfirstlane(nth_expert(choices.used, n));
    up_tile<DT, EPI, MANY>(a, scalar(choices.weights[0][expert]), scalar(choices.weights[1][expert]), false, unit % tiles, tokens_of(a, choices, expert), lds);
}

// The gate, beside which the shared expert's tiles run, as they wait for nothing.  A block takes TT tokens and 4 experts: products and sums in 64 bits, as in moe_route, every
// lane 8 neighbouring elements, the waves share out the row in chunks of 512.  The block that brings a tile of tokens its last logits selects for it, a wave per token.
// 64 experts and one token of 2048, beside a shared expert of 2 x 2816 columns (23 MB), 8.7 us.  (Selection by every block of `up` from the logits, up to four tokens: 13.7 instead
// of 14.0 us for one token of the smallest layer, 47.3 instead of 45.6 where a shared expert's tiles take longer than the selection.)
template <int DT, int EPI, int TT, bool MANY>
__global__ __launch_bounds__(64 * kFewWaves) void few_gate_kernel(const FewArgs a) {
    constexpr int B = DT == MOE_BF16 ? 2 : 4, NQ = B / 2;
    __shared__ float lds[kUpLds<EPI, MANY>];
    __shared__ double part[kFewWaves][TT * 4];
    __shared__ int flag;
    clear_done(a);
    const int tiles_e = (a.E + 3) / 4, tiles_t = (a.T + TT - 1) / TT;
    if ((int)blockIdx.x >= tiles_e * tiles_t) return shared_tile<DT, EPI, MANY>(a, blockIdx.x - tiles_e * tiles_t, lds);
    const int tile = blockIdx.x / tiles_e, t0 = tile * TT, e0 = blockIdx.x % tiles_e * 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t bytes = (uint32_t)a.H * B;
    auto row = [&](const void* p, int r) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(p)) + (size_t)r * bytes, 0, bytes, 0x00027000); };
    double sum[TT][4] = {};
    for (int c = wave; c * 512 < a.H; c += kFewWaves) {
        const int at = (c * 512 + lane * 8) * B;             // past the row's end: zeros
        u32x4 xq[TT][NQ], wq[4][NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) wq[e][q] = __builtin_amdgcn_raw_buffer_load_b128(row(a.gate, min(e0 + e, a.E - 1)), at + 16 * q, 0, 0);
#pragma unroll
            for (int t = 0; t < TT; ++t) xq[t][q] = __builtin_amdgcn_raw_buffer_load_b128(row(a.x, min(t0 + t, a.T - 1)), at + 16 * q, 0, 0);
        }
        auto value = [](const u32x4 (&v)[NQ], int j) {
            if (DT == MOE_BF16) return (double)(j & 1 ? __uint_as_float(v[0][j / 2] & 0xffff0000u) : bf16_bits_to_f32(v[0][j / 2] & 0xffffu));
            return (double)__uint_as_float(v[j / 4 % NQ][j % 4]);
        };
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            double xv[TT], wv[4];
#pragma unroll
            for (int t = 0; t < TT; ++t) xv[t] = value(xq[t], j);
#pragma unroll
            for (int e = 0; e < 4; ++e) wv[e] = value(wq[e], j);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[t][e] = __builtin_fma(xv[t], wv[e], sum[t][e]);
        }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double v = wave_sum(sum[t][e]);
            if (lane == 0) part[wave][t * 4 + e] = v;
        }
    __syncthreads();
    const int i = threadIdx.x, t = t0 + i / 4, e = e0 + i % 4;
    if (i < TT * 4 && t < a.T && e < a.E) {
        double v = a.gate_bias ? (double)a.gate_bias[e] : 0.0;
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) s += part[w][i];
        v += s;
        const uint2 u = __builtin_bit_cast(uint2, v);
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{u.x, u.y}, all_of(a.logits), (t * a.E + e) * 8, 0, kAgentScope);
    }
    if (!last_piece(a.gate_done + tile, tiles_e, &flag)) return;
    if (threadIdx.x == 0) __hip_atomic_store(a.gate_done + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
    if (wave >= TT || t0 + wave >= a.T) return;
    const Choice c = select(a, [&](int e) {
        const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(all_of(a.logits), e < a.E ? ((t0 + wave) * a.E + e) * 8 : 0x80000000u, 0, kAgentScope);
        return __builtin_bit_cast(double, uint2{u[0], u[1]});
    });
    if (lane < a.k) {
        a.idx[(t0 + wave) * a.k + lane] = c.expert;
        a.w[(t0 + wave) * a.k + lane] = c.weight;
    }
}

// 16 columns of an expert for its tokens, in bf16 layers both parts of eight tokens a tile, so that a product of 16 columns takes both.  MANY: more than 16 tokens
// The layers above: 199 us (0.94 GB, 4.7 TB/s), 14 us (46 MB).  All experts of 16 columns by one block, without partial sums, keep too few bytes on their way: 25 to 126 us where this
// takes 14 to 18.
template <int DT, bool MANY>
__global__ __launch_bounds__(64 * kFewWaves, MANY ? 3 : 4) void few_down_kernel(const FewArgs a) {
    constexpr int B = DT == MOE_BF16 ? 2 : 4, TILE = DT == MOE_BF16 ? 8 : 16, MOST = (MANY ? kFewTokens : 16) / TILE;
    __shared__ Choices choices;
    __shared__ float lds[MOST * kFewWaves * 256];
    __shared__ int flag;
    read_choices(a, choices);
    const int tiles = (a.H + 15) / 16, tile = blockIdx.x % tiles, unit = blockIdx.x / tiles, lane = threadIdx.x & 63;
    const int has_shared = a.F_shared > 0 ? 1 : 0, units = __builtin_popcountll(choices.used) + has_shared;
    if (unit >= max(units, 1)) return;
    const __amdgpu_buffer_rsrc_t parts = pieces_rsrc(a.parts, 0x7fffffffu);
    if (units > 0) {
        const bool shared = unit < has_shared;
        const int expert = shared ? 0 : __builtin_amdgcn_readfirstlane(nth_expert(choices.used, unit - has_shared)), width = shared ? a.F_shared : a.F;
        const Tokens tok = shared ? all_tokens(a) : tokens_of(a, choices, expert);
        const uint32_t bytes = (uint32_t)width * B, rest = (uint32_t)(shared ? a.T : a.T * a.k) * bytes;   // from a row to what its rounding leaves
        const char* const here = scalar(choices.weights[2][expert]);   // (not in the choice below: one address of two kinds of memory would make it a FLAT load)
        const char* const w[1] = {(shared ? reinterpret_cast<const char*>(a.s_down) : here) + (size_t)tile * 16 * bytes};
        const int last = min(15, a.H - 1 - tile * 16);
        float weight = 1.f;                                  // of the lane's token: all of its choices of the expert
        if (!shared) {
            weight = 0.f;
            for (int q = tok.row; q < (tok.token + 1) * a.k; ++q) weight += choices.at[q] == expert ? choices.by[q] : 0.f;
        }
        auto run = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            uint32_t row_off[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                row_off[t] = (uint32_t)__shfl(tok.row, min(TILE * t + (lane & (TILE - 1)), tok.count - 1), 64) * bytes + (TILE == 8 && (lane & 8) ? rest : 0u);
                asm volatile("" : "+v"(row_off[t]));         // (the multiplication gives 64 bits, whose upper half would keep a register through the loop)
            }
            float v[1][NT];
            block_sums<DT, 1, NT, TILE == 8>(w, last, bytes, all_of(shared ? a.h_shared : a.h), row_off, lds, v);
            const int i = threadIdx.x, row = 4 * (i >> 6) + (i & 3), col = (i >> 2) & 15;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int place = TILE * t + col, to = __shfl(tok.row, place & 63, 64) + (shared ? a.T * a.k : 0);
                const float f = v[0][t] * __shfl(weight, place & 63, 64);
                if (col < TILE && place < tok.count && row <= last) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(f), parts, ((uint32_t)to * a.H + tile * 16 + row) * 4, 0, kAgentScope);
            }
        };
        if (MOST == 1 || tok.count <= TILE) run(std::integral_constant<int, 1>{});
        else if (MOST == 2 || tok.count <= 2 * TILE) run(std::integral_constant<int, MOST < 2 ? 1 : 2>{});
        else if (MOST == 4 || tok.count <= 4 * TILE) run(std::integral_constant<int, MOST < 4 ? 1 : 4>{});
        else run(std::integral_constant<int, MOST < 8 ? 1 : 8>{});
        if (!last_piece(a.done + tile, units, &flag)) return;
    }
    // of a token's choices of one expert, which share a row, the first alone counts
    for (int i = threadIdx.x; i < a.T * a.k; i += 64 * kFewWaves) {
        bool first = true;
        for (int q = i - i % a.k; q < i; ++q) first = first && choices.at[q] != choices.at[i];
        if (!first) choices.at[i] = -1;                      // (those that look for it find the first)
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 4; i += 64 * kFewWaves) {   // four columns of a token
        const int t = i / 4, col = tile * 16 + i % 4 * 4;
        if (col >= a.H) continue;
        auto part = [&](int row, bool there) {
            return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, there ? ((uint32_t)row * a.H + col) * 4 : 0x80000000u, 0, kAgentScope));
        };
        f32x4 v = {0.f, 0.f, 0.f, 0.f}, last = part(a.T * a.k + t, has_shared);
        constexpr int AHEAD = MANY ? 4 : 8;                  // on their way at a time
        for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
            f32x4 u[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) u[j] = part(t * a.k + j0 + j, j0 + j < a.k && choices.at[t * a.k + min(j0 + j, a.k - 1)] >= 0);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) v += u[j];       // (zeros where there is none)
        }
        v += last;
        if (DT == MOE_BF16) *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.y) + (size_t)t * a.H + col) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.y) + (size_t)t * a.H + col) = v;
    }
}

// A layer of small experts: a block per token does all of it, in one launch instead of three.  Sixteen lanes share a row of weights, 16 bytes each at a time, for several rows at once; x, the
// logits and the inner activations (in fp32) stay in LDS.  One CU's loads and arithmetic for a token: bound by launch and round trips, from 100 thousand elements on by the latter.
// bf16, one token and 64 of them (three launches): 128 -> 128, two of eight, 66 thousand elements 7.8 and 8.1 us (13.1, 20.6); 256 -> 256, 264 thousand 11.5 and 12.1 (13.1, 21.5), fp32 13.5
// and 17.1 (13.7, 22.2); 128 -> 512 SwiGLU, 394 thousand 18.9 and 19.6 (13.5, 22.0).  The choice does not look at T, so that a token's result is the same in any batch.  With 8 waves a
// block 13.8 instead of 11.5.
constexpr int kSmallWaves = 16, kSmallWidth = 2048, kSmallInner = 4096;
constexpr size_t kSmallElements = 1 << 18;                   // of weights that a token takes
typedef const __attribute__((address_space(1))) u32x4* GlobalQ;   // (addresses from LDS tables: else they are accessed by FLAT instructions)
template <int DT, class T, int R> __device__ __forceinline__ void small_dot(const uint64_t (&row)[R], const float* v, int n, T (&sum)[R], T weight) {
    constexpr int V = DT == MOE_BF16 ? 8 : 4;                // of 16 bytes
    T s[R] = {};
    for (int i = (threadIdx.x & 15) * V; i < n; i += 16 * V) {
        u32x4 q[R];
#pragma unroll
        for (int r = 0; r < R; ++r) q[r] = *reinterpret_cast<GlobalQ>(row[r] + (size_t)i * (16 / V));
        float x[V];
#pragma unroll
        for (int j = 0; j < V; j += 4) *reinterpret_cast<f32x4*>(x + j) = *reinterpret_cast<const f32x4*>(v + i + j);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float w = DT == MOE_BF16 ? (j & 1 ? __uint_as_float(q[r][j / 2] & 0xffff0000u) : bf16_bits_to_f32(q[r][j / 2] & 0xffffu)) : __uint_as_float(q[r][j % 4]);
                s[r] = __builtin_elementwise_fma((T)w, (T)x[j], s[r]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = __builtin_elementwise_fma(weight, s[r], sum[r]);
}
template <class T> __device__ __forceinline__ T sum_of_16(T v) {
    auto turn = [](T u, auto ctrl) {
        constexpr int C = decltype(ctrl)::value;
        if constexpr (sizeof(T) == 8) return ror<C>(u);
        else return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(u), C, 0xF, 0xF, true));
    };
    v += turn(v, std::integral_constant<int, 0x128>{}); v += turn(v, std::integral_constant<int, 0x124>{});
    v += turn(v, std::integral_constant<int, 0x122>{}); return v + turn(v, std::integral_constant<int, 0x121>{});
}
template <int DT, int EPI>
__global__ __launch_bounds__(64 * kSmallWaves) void few_small_kernel(const FewArgs a) {
    constexpr int B = DT == MOE_BF16 ? 2 : 4, V = 16 / B, GROUPS = 4 * kSmallWaves, R = 4, NF = EPI == EPI_SWIGLU ? 2 : 1;
    __shared__ f32x4 x_lds[kSmallWidth / 4], h_lds[kSmallInner / 4];
    __shared__ double logits[MOE_MAX_E];
    __shared__ uint32_t local[MOE_MAX_E / 4];
    __shared__ uint64_t weights[3][MOE_MAX_LOCAL + 1];       // the shared expert behind the others
    __shared__ int place[MOE_MAX_K];
    __shared__ float by[MOE_MAX_K];
    float *const x = reinterpret_cast<float*>(x_lds), *const h = reinterpret_cast<float*>(h_lds);
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, group = tid >> 4;
    auto address = [](const void* p) { return (uint64_t)reinterpret_cast<uintptr_t>(p); };
    for (int i = tid * V; i < a.H; i += 64 * kSmallWaves * V) {
        const u32x4 q = *reinterpret_cast<GlobalQ>(address(a.x) + ((size_t)t * a.H + i) * B);
#pragma unroll
        for (int j = 0; j < V; ++j) x[i + j] = DT == MOE_BF16 ? (j & 1 ? __uint_as_float(q[j / 2] & 0xffff0000u) : bf16_bits_to_f32(q[j / 2] & 0xffffu)) : __uint_as_float(q[j % 4]);
    }
    if (tid < MOE_MAX_E / 4) local[tid] = reinterpret_cast<const uint32_t*>(a.local)[tid];
    if (tid <= MOE_MAX_LOCAL) {
        const bool shared = tid == MOE_MAX_LOCAL;
        const int e = min(tid, MOE_MAX_LOCAL - 1);
        const void *const w0 = a.tab.w1[e], *const w1 = a.tab.w_up[e], *const w2 = a.tab.w_down[e];
        weights[0][tid] = address(shared ? a.s1 : w0);
        weights[1][tid] = address(shared ? a.s_up : w1);
        weights[2][tid] = address(shared ? a.s_down : w2);
    }
    if (!a.gate && tid < a.k) {
        place[tid] = a.idx[t * a.k + tid];
        by[tid] = a.w[t * a.k + tid];
    }
    __syncthreads();
    if (a.gate) {
        for (int e0 = group; e0 < a.E; e0 += GROUPS * R) {
            uint64_t row[R];
            double z[R] = {};
#pragma unroll
            for (int r = 0; r < R; ++r) row[r] = address(a.gate) + (size_t)min(e0 + GROUPS * r, a.E - 1) * a.H * B;
            small_dot<DT, double, R>(row, x, a.H, z, 1.0);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int e = e0 + GROUPS * r;
                const double v = sum_of_16(z[r]);
                if ((tid & 15) == 0 && e < a.E) logits[e] = (a.gate_bias ? (double)a.gate_bias[e] : 0.0) + v;
            }
        }
        __syncthreads();
        if (tid < 64) {
            const Choice c = select(a, [&](int e) { return logits[min(e, a.E - 1)]; });
            if (lane < a.k) {
                a.idx[t * a.k + lane] = c.expert;
                a.w[t * a.k + lane] = c.weight;
                place[lane] = c.expert;
                by[lane] = c.weight;
            }
        }
        __syncthreads();
    }
    // place: from here on that of the table, -1: not here
    int mine = -1;
    if (tid < a.k) mine = (unsigned)place[tid] < (unsigned)a.E ? reinterpret_cast<const int8_t*>(local)[place[tid]] : -1;
    __syncthreads();
    if (tid < a.k) place[tid] = mine;
    __syncthreads();
    const int routed = a.k * a.F, rows = routed + a.F_shared;
    for (int f0 = group; f0 < rows; f0 += GROUPS * R) {
        uint64_t row[NF][R];
        float s[NF][R] = {};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = min(f0 + GROUPS * r, rows - 1), j = min(i / a.F, a.k - 1), e = i < routed ? place[j] : MOE_MAX_LOCAL;
            // (of an expert that is not here: some row that is, the one that is read for it)
#pragma unroll
            for (int f = 0; f < NF; ++f) row[f][r] = e >= 0 ? weights[f][e] + (size_t)(i < routed ? i - j * a.F : i - routed) * a.H * B : address(a.x) + (size_t)t * a.H * B;
        }
#pragma unroll
        for (int f = 0; f < NF; ++f) small_dot<DT, float, R>(row[f], x, a.H, s[f], 1.f);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = f0 + GROUPS * r;
            const float g = sum_of_16(s[0][r]), u = sum_of_16(s[NF - 1][r]);
            if ((tid & 15) == 0 && i < rows) h[i] = activation_fast<EPI>(g, NF == 2 ? u : 0.f);
        }
    }
    __syncthreads();
    for (int c0 = group; c0 < a.H; c0 += GROUPS * R) {
        float v[R] = {};
        auto add = [&](int e, const float* from, int width, float weight) {
            uint64_t row[R];
#pragma unroll
            for (int r = 0; r < R; ++r) row[r] = weights[2][e] + (size_t)min(c0 + GROUPS * r, a.H - 1) * width * B;
            small_dot<DT, float, R>(row, from, width, v, weight);
        };
        for (int j = 0; j < a.k; ++j)
            if (place[j] >= 0) add(place[j], h + j * a.F, a.F, by[j]);
        if (a.F_shared) add(MOE_MAX_LOCAL, h + routed, a.F_shared, 1.f);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = c0 + GROUPS * r;
            const float f = sum_of_16(v[r]);
            if ((tid & 15) != 0 || c >= a.H) continue;
            if (DT == MOE_BF16) reinterpret_cast<uint16_t*>(a.y)[(size_t)t * a.H + c] = (uint16_t)f32_to_bf16_bits(f);
            else reinterpret_cast<float*>(a.y)[(size_t)t * a.H + c] = f;
        }
    }
}
bool is_small(const moe_shape& s, int F, int F_shared, int act) {
    const size_t inner = (size_t)s.k * F + F_shared, elements = (size_t)s.H * (s.E + inner * (act == MOE_ACT_SWIGLU ? 3 : 2));
    return s.H <= kSmallWidth && inner <= (size_t)kSmallInner && elements <= kSmallElements;
}

struct FewSpace { size_t h, h_shared, parts, logits, done, bytes; };
FewSpace few_space(const moe_shape& s, int F, int F_shared) {
    FewSpace p;
    p.h = 0;                                                 // 4 bytes an element: fp32, or two of bf16
    p.h_shared = align256((size_t)s.T * s.k * F * 4);
    p.parts = p.h_shared + align256((size_t)s.T * F_shared * 4);
    p.logits = p.parts + align256((size_t)s.T * (s.k + 1) * s.H * 4);
    p.done = p.logits + align256((size_t)s.T * s.E * 8);
    p.bytes = p.done + align256((size_t)(s.H + 15) / 16 * 4);
    return p;
}
bool few_sizes_ok(const moe_shape& s, int F, int F_shared) {
    const int unit = s.dtype == MOE_BF16 ? 128 : 4;
    return F > 0 && F_shared >= 0 && s.H % unit == 0 && F % unit == 0 && F_shared % unit == 0 && s.H <= kFewWidth && F <= kFewWidth && F_shared <= kFewWidth;
}

// A context's counters before its first gate, on the call's own stream: the context's creation would have to wait for it, and so for whatever else runs.  In a graph
// that is captured before any call has run, the kernel is recorded with the others; the next call that runs clears once more.
__global__ __launch_bounds__(MOE_GATE_TILES) void few_clear_kernel(int32_t* gate_done) { gate_done[threadIdx.x] = 0; }
int clear_gate(moe_ctx* ctx, hipStream_t st) {
    if (ctx->gate_clear) return MOE_OK;
    hipStreamCaptureStatus capture;
    MOE_HIP(hipStreamIsCapturing(st, &capture));
    hipLaunchKernelGGL(few_clear_kernel, dim3(1), dim3(MOE_GATE_TILES), 0, st, ctx->gate_done);
    MOE_LAUNCH_CHECK("few_clear_kernel");
    ctx->gate_clear = capture == hipStreamCaptureStatusNone;
    return MOE_OK;
}

template <int DT, int EPI, bool MANY> int launch_few(FewArgs a, int slots, hipStream_t st) {
    const dim3 threads(64 * kFewWaves);
    const int shared_tiles = (a.F_shared + 15) / 16;
    a.shared_here = a.clear = 1;
    if (a.gate) {
        if (a.T == 1) hipLaunchKernelGGL((few_gate_kernel<DT, EPI, 1, false>), dim3((a.E + 3) / 4 + shared_tiles), threads, 0, st, a);
        else hipLaunchKernelGGL((few_gate_kernel<DT, EPI, 4, MANY>), dim3((a.E + 3) / 4 * ((a.T + 3) / 4) + shared_tiles), threads, 0, st, a);
        MOE_LAUNCH_CHECK("few_gate_kernel");
        a.shared_here = a.clear = 0;
    }
    const int up = (a.shared_here ? shared_tiles : 0) + (a.F + 15) / 16 * slots;
    if (up > 0) {
        hipLaunchKernelGGL((few_up_kernel<DT, EPI, MANY>), dim3(up), threads, 0, st, a);
        MOE_LAUNCH_CHECK("few_up_kernel");
    }
    hipLaunchKernelGGL((few_down_kernel<DT, MANY>), dim3((a.H + 15) / 16 * std::max(1, slots + (a.F_shared > 0 ? 1 : 0))), threads, 0, st, a);
    MOE_LAUNCH_CHECK("few_down_kernel");
    return MOE_OK;
}
template <int DT> int launch_few(const FewArgs& a, int act, int slots, bool small, hipStream_t st) {
    if (small) {
        const dim3 grid(a.T), threads(64 * kSmallWaves);
        if (act == MOE_ACT_SWIGLU) hipLaunchKernelGGL((few_small_kernel<DT, EPI_SWIGLU>), grid, threads, 0, st, a);
        else if (act == MOE_ACT_GELU_MLP) hipLaunchKernelGGL((few_small_kernel<DT, EPI_GELU>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((few_small_kernel<DT, EPI_SILU>), grid, threads, 0, st, a);
        MOE_LAUNCH_CHECK("few_small_kernel");
        return MOE_OK;
    }
#define MOE_FEW(EPI) return a.T > 16 ? launch_few<DT, EPI, true>(a, slots, st) : launch_few<DT, EPI, false>(a, slots, st)
    if (act == MOE_ACT_SWIGLU) MOE_FEW(EPI_SWIGLU);
    if (act == MOE_ACT_GELU_MLP) MOE_FEW(EPI_GELU);
    MOE_FEW(EPI_SILU);
#undef MOE_FEW
}

}  // namespace

extern "C" size_t moe_layer_few_workspace_bytes(const moe_ctx* ctx, int32_t F, int32_t F_shared) {
    return ctx && ctx->s.T <= kFewTokens && few_sizes_ok(ctx->s, F, F_shared) ? few_space(ctx->s, F, F_shared).bytes : 0;
}

extern "C" int moe_layer_few(moe_ctx* ctx, const void* x, const void* Wg, const float* gate_bias, int32_t* topk_idx, float* topk_w, const moe_expert_w* experts,
                             int32_t n_local, const int32_t* expert_local, int32_t F, int32_t act, const moe_expert_w* shared, int32_t F_shared, void* y, void* workspace,
                             size_t workspace_bytes, void* stream) {
    if (!ctx || !x || !topk_idx || !topk_w || (n_local != 0 && !experts) || !expert_local || !y || !workspace) return moe_set_error(MOE_EINVAL, "moe_layer_few: NULL argument");
    const moe_shape& s = ctx->s;
    if (n_local < 0 || F <= 0 || F_shared < 0) return moe_set_error(MOE_EINVAL, "moe_layer_few: negative size");
    if ((shared != nullptr) != (F_shared > 0)) return moe_set_error(MOE_EINVAL, "moe_layer_few: F_shared > 0 goes with a shared expert");
    if (!Wg && gate_bias) return moe_set_error(MOE_EINVAL, "moe_layer_few: gate_bias without Wg");
    if (act < 0 || act > 2) return moe_set_error(MOE_EDTYPE, "moe_layer_few: unknown act %d", act);
    if (s.T > kFewTokens) return moe_set_error(MOE_ESHAPE, "moe_layer_few: T <= %d required", kFewTokens);
    if (s.capacity != 0) return moe_set_error(MOE_ESHAPE, "moe_layer_few: a context without capacity required");
    if (n_local > MOE_MAX_LOCAL) return moe_set_error(MOE_ESHAPE, "moe_layer_few: n_local <= %d required", MOE_MAX_LOCAL);
    if (!few_sizes_ok(s, F, F_shared))
        return moe_set_error(MOE_ESHAPE, "moe_layer_few: H, F and F_shared must be multiples of %d and at most %d", s.dtype == MOE_BF16 ? 128 : 4, kFewWidth);
    if (!aligned16(x) || !aligned16(Wg) || !aligned16(y) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return moe_set_error(MOE_EALIGN, "moe_layer_few: x, Wg and y need 16-byte, workspace 256-byte alignment");
    const FewSpace p = few_space(s, F, F_shared);
    if (workspace_bytes < p.bytes) return moe_set_error(MOE_ESHAPE, "moe_layer_few: workspace too small (%zu < %zu)", workspace_bytes, p.bytes);
    FewArgs a = {};
    unsigned long long seen = 0;
    for (int e = 0; e < s.E; ++e) {
        const int at = expert_local[e];
        if (at < -1 || at >= n_local) return moe_set_error(MOE_ESHAPE, "moe_layer_few: expert_local[%d] = %d is outside [-1, %d)", e, at, n_local);
        if (at >= 0 && (seen >> at & 1)) return moe_set_error(MOE_ESHAPE, "moe_layer_few: two experts at place %d", at);
        if (at >= 0) seen |= 1ull << at;
        a.local[e] = (int8_t)at;
    }
    for (int e = 0; e < n_local + (shared ? 1 : 0); ++e) {
        const moe_expert_w& w = e < n_local ? experts[e] : *shared;
        if (!w.w1 || !w.w_down || (act == MOE_ACT_SWIGLU && !w.w_up)) return moe_set_error(MOE_EINVAL, "moe_layer_few: expert %d has a NULL weight", e);
        if (!aligned16(w.w1) || !aligned16(w.w_up) || !aligned16(w.w_down)) return moe_set_error(MOE_EALIGN, "moe_layer_few: expert %d weights must be 16-byte aligned", e);
        if (e == n_local) {
            a.s1 = w.w1; a.s_up = w.w_up; a.s_down = w.w_down;
        } else {
            a.tab.w1[e] = w.w1; a.tab.w_up[e] = w.w_up; a.tab.w_down[e] = w.w_down;
        }
    }
    if (Wg) ctx->rank_src = nullptr;                         // the indices are about to change
    char* const ws = reinterpret_cast<char*>(workspace);
    a.x = x; a.idx = topk_idx; a.w = topk_w; a.y = y;
    a.h = ws + p.h; a.h_shared = ws + p.h_shared;
    a.gate = Wg; a.gate_bias = gate_bias; a.gate_done = ctx->gate_done; a.renorm = s.renorm;
    a.logits = reinterpret_cast<double*>(ws + p.logits);
    a.parts = reinterpret_cast<float*>(ws + p.parts);
    a.done = reinterpret_cast<int32_t*>(ws + p.done);
    a.T = s.T; a.H = s.H; a.F = F; a.F_shared = F_shared; a.E = s.E; a.k = s.k;
    const int slots = std::min(s.T * s.k, n_local);          // experts in use, at most
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool small = is_small(s, F, F_shared, act);
    if (Wg && !small)
        if (const int rc = clear_gate(ctx, st)) return rc;
    return s.dtype == MOE_BF16 ? launch_few<MOE_BF16>(a, act, slots, small, st) : launch_few<MOE_F32>(a, act, slots, small, st);
}
