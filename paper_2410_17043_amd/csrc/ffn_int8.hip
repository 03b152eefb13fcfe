// Expert FFN in 8-bit integers (a scale per received row and per output channel of a weight), a ragged grouped GEMM pair with the quantisation of what lies between.
//
//   GEMM1   h = act(s_r s_1 (q_r . W1^T) [, s_r s_up (q_r . Wu^T)]), rounded to bf16
//   rows    of h quantised again: q = h / s, s = max |h| / 127
//   GEMM2   out = s s_down (q . Wd^T), bf16
//
// v_mfma_i32_16x16x64_i8: products and their sums are exact, so no result depends on tiles, on cuts along K or on other rows; the scales are
// applied once, behind the sum, in fp32.  A row's scale needs its whole row of h, which many blocks make, so h goes through memory in bf16 (a row is then read twice as bytes of
// half: 0.15 ms of the 2.95 of the largest share; quantised on their way to LDS in the second GEMM of few rows, 16 numbers a thread and stage in 64 bits, that GEMM took 25 us instead of
// 17 and 5).  The map of tiles is that of the bf16 kernels (ffn_tiles.h), their shapes and choice those of the e4m3 ones (ffn_tiles8.h).
#include "ffn_tiles8.h"
#include "int8.h"
#include <type_traits>

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kBlockK = 128;                                 // bytes of K of a trip

struct ExpertTableI {
    const void *w1[MOE_MAX_LOCAL], *w_up[MOE_MAX_LOCAL], *w_down[MOE_MAX_LOCAL];
    const float *s1[MOE_MAX_LOCAL], *s_up[MOE_MAX_LOCAL], *s_down[MOE_MAX_LOCAL];
};

__device__ __forceinline__ int from_agpr_i(int a) {
    int v;
    asm("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
    return v;
}

// ------------------------------------------------------------------------------------ rows
// W waves per row, CH loads of 16 bytes a lane, all of which go out before any is used; a block is 4 / W rows, one for W >= 4.  Longer rows (CH = 0) are read twice, the second time
// from the caches.  Bound by memory: 20571 rows of 14336 in bf16 150 us (885 MB, 5.9 TB/s; read twice it was 207), in fp32 274 (1475 MB, 5.4 TB/s); 16384 of 2048 in fp32 30.5 us.
template <int DT, int CH>
__global__ __launch_bounds__(512) void quantize_int8_kernel(const void* __restrict__ x, int T, int H, uint8_t* __restrict__ rows, int pitch, int W) {
    __shared__ uint32_t part[8];
    constexpr int B = DT == MOE_BF16 ? 2 : 4, V = 16 / B;    // elements of a load; H is a multiple of 128
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = wave / W * W, step = W * 64;
    const int row = blockIdx.x * (W < 4 ? 4 / W : 1) + wave / W, at = (wave - first) * 64 + lane, t = min(row, T - 1);
    const __amdgpu_buffer_rsrc_t in = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(x)) + (size_t)t * H * B, 0, (uint32_t)H * B, 0x00027000);
    auto load = [&](int i) { return __builtin_amdgcn_raw_buffer_load_b128(in, i * 16, 0, 0); };   // behind the row's end: zeros
    auto element = [](const u32x4& q, int j) { return DT == MOE_BF16 ? (j & 1 ? __uint_as_float(q[j / 2] & 0xffff0000u) : bf16_bits_to_f32(q[j / 2] & 0xffffu)) : __uint_as_float(q[j % 4]); };
    uint32_t most = 0;
    auto look = [&](const u32x4& q) {
#pragma unroll
        for (int j = 0; j < V; ++j) most = max(most, abs_bits(element(q, j)));
    };
    u32x4 held[CH + 1];
    if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) held[c] = load(c * step + at);
#pragma unroll
        for (int c = 0; c < CH; ++c) look(held[c]);
    } else {
        for (int i = at; i < H / V; i += step) look(load(i));
    }
    most = max_of_16_lanes(most);
    most = max(max(__builtin_amdgcn_readlane(most, 0), __builtin_amdgcn_readlane(most, 16)), max(__builtin_amdgcn_readlane(most, 32), __builtin_amdgcn_readlane(most, 48)));
    if (W > 1) {
        if (lane == 0) part[wave] = most;
        __syncthreads();
        most = __builtin_amdgcn_readlane(max_of_16_lanes((lane & 15) < W ? part[first + (lane & 7)] : 0u), 0);
    }
    if (row >= T) return;
    const Int8Scale s = int8_scale((double)__uint_as_float(most));
    uint8_t* const out = rows + (size_t)row * pitch;
    auto put = [&](int i, const u32x4& q) {
        if (i >= H / V) return;
        uint32_t b[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j)
            b[j] = s.inverse == 0.0 ? 0u : int8_pack4<DT == MOE_F32>(element(q, 4 * j), element(q, 4 * j + 1), element(q, 4 * j + 2), element(q, 4 * j + 3), s.inverse);
        if (V == 8) *reinterpret_cast<u32x2*>(out + i * 8) = u32x2{b[0], b[V / 4 - 1]};
        else *reinterpret_cast<uint32_t*>(out + i * 4) = b[0];
    };
    if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) put(c * step + at, held[c]);
    } else {
        for (int i = at; i < H / V; i += step) put(i, load(i));
    }
    if (wave == first && lane < (pitch - H) / 4) *reinterpret_cast<uint32_t*>(out + H + 4 * lane) = lane == 0 ? __float_as_uint(s.s) : 0u;
}
template <int DT> int launch_quantize(const void* x, int64_t T, int H, uint8_t* rows, hipStream_t st) {
    const int loads = H * (DT == MOE_BF16 ? 2 : 4) / 1024 + 1;   // of a wave, at most
    const int W = loads <= 2 ? 1 : loads <= 4 ? 2 : loads <= 16 ? 4 : 8, CH = (loads + W - 1) / W, pitch = (int)int8_row_bytes(H);
    const int64_t most = ((int64_t)1 << 31) / (64 * W);      // of 2^32 threads and more only the number modulo 2^32 would run
    for (int64_t t = 0; t < T; t += most) {
        const int n = (int)std::min(most, T - t);
        const dim3 grid(W < 4 ? (n * W + 3) / 4 : n), threads(W < 4 ? 256 : 64 * W);
        const char* const from = reinterpret_cast<const char*>(x) + (size_t)t * H * (DT == MOE_BF16 ? 2 : 4);
        uint8_t* const to = rows + (size_t)t * pitch;
        if (CH <= 2) hipLaunchKernelGGL((quantize_int8_kernel<DT, 2>), grid, threads, 0, st, from, n, H, to, pitch, W);
        else if (CH <= 4) hipLaunchKernelGGL((quantize_int8_kernel<DT, 4>), grid, threads, 0, st, from, n, H, to, pitch, W);
        else if (CH <= 8) hipLaunchKernelGGL((quantize_int8_kernel<DT, 8>), grid, threads, 0, st, from, n, H, to, pitch, W);
        else hipLaunchKernelGGL((quantize_int8_kernel<DT, 0>), grid, threads, 0, st, from, n, H, to, pitch, W);
        MOE_LAUNCH_CHECK("quantize_int8_kernel");
    }
    return MOE_OK;
}

// ------------------------------------------------------------------------------------ tiles
// The scale of a received row r of a tile (the last one that there is for those behind it)
__device__ __forceinline__ float row_scale(const uint8_t* A, int lda, int K, const Item8& t, int r) {
    const int c = min(r, t.nrows - 1);
    return *reinterpret_cast<const float*>(A + (size_t)(t.row0 + (t.rel ? t.rel[c] : c)) * lda + K);
}

// Stores of a wave's part of a tile, NI tiles of 16 rows by NJ tiles of 16 columns, as bf16.  value(i, j, e, factor(i)): row 16 i + lane % 16, column 16 j + 4 (lane / 16) + e.  Four
// neighbouring columns of a row are one 8-byte piece; 32 rows at a time cross LDS (`region`, this wave's own 4 KB) and leave as whole lines.  Chunk c (16 bytes) of
// row r lies at slot c ^ (r / 2): writes of 32 lanes and reads of 16 fall on all banks once.
template <int NI, int NJ, class Value, class Factor>
__device__ __forceinline__ void store_rows(Value value, Factor factor, int lane, unsigned char* region, __amdgpu_buffer_rsrc_t dst, int first_row, const Item8& t, int ldc) {
    const int r = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int i = 0; i < NI; i += 2) {
        const float of_row[2] = {factor(i), factor(i + 1)};
        uint32_t off[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) off[it] = row_offset(t, first_row + 16 * i + 8 * it + (lane >> 3), ldc) + (lane & 7) * 16;
#pragma unroll
        for (int p = 0; p < NJ / 4; ++p) {                   // 64 columns
            asm volatile("" ::: "memory");
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = 16 * h + r;
                    auto v = [&](int e) { return value(i + h, 4 * p + j, e, of_row[h]); };
                    *reinterpret_cast<u32x2*>(region + row * 128 + (((2 * j + (quarter >> 1)) ^ ((row >> 1) & 7)) << 4) + ((quarter & 1) << 3)) = u32x2{pack_bf16(v(0), v(1)), pack_bf16(v(2), v(3))};
                }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int rr = 8 * it + (lane >> 3);
                const u32x4 q = *reinterpret_cast<const u32x4*>(region + rr * 128 + (((lane & 7) ^ ((rr >> 1) & 7)) << 4));
                __builtin_amdgcn_raw_buffer_store_b128(q, dst, off[it], p * 128, 0);
            }
        }
    }
}

// C = epilogue(A . B^T) for one tile of 64 MI rows and 64 NJ weight rows.  SwiGLU: the weight rows are, per wave column wn (16 NJ output
// columns), 16 NJ rows of W1 followed by the 16 NJ rows of Wu for the same columns, so that a lane has the gate and the up product of a column.
//
// Pipeline, as in the e4m3 kernels: 2 P + 1 stages of 64 bytes of K, loads straight to LDS in pairs of stages, spread between the products, fragments read a stage ahead, one
// barrier per stage; the pipeline runs on across the tiles that a block walks through.  A fragment is 16 rows x 64 bytes of K, 16 bytes in a lane, and the products of 16 x 16 x 64 go in
// runs with the weights' operand in common: bound by power, which lets these sustain 3.82 POP/s from registers and those of 32 x 32 x 32 3.50.  20571 rows of 4096 -> 14336 -> 4096,
// SwiGLU: 1.96 ms (2.46 POP/s) and 0.86 ms (2.8 POP/s) with the sum of the cut tiles, 256 x 256 each; 2741 rows of six experts, 1152 -> 2304 -> 1152: 18.5 and 15 us.
template <int EPI, int MI, int NJ, int P, bool CUT>
__global__ __launch_bounds__(256, (Geom8<MI, NJ, P>::PER_CU)) void gemm_int8_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTableI tab, int which0, int which1, int N, int K,
                                                          char* __restrict__ C, int ldc, int tiles_n, int ncu, int walk, int most_cut, int* pieces) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    using TG = Geom8<MI, NJ, P>;
    using OG = Out8<EPI, NJ>;
    constexpr int LOADS = 2 * (MI + NJ), FIRST = MI + NJ;    // loads per pair of stages and wave; those in the first half of a trip
    constexpr int OPEN = (P - 2) * LOADS + FIRST;            // loads that may be outstanding in the middle of a trip: those of pairs that are needed later
    static_assert(OPEN < 64 && P >= 2, "");
    auto word = [](const int32_t* p) { return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p)); };
    const int n_tiles_m = word(m.n_tiles);
    const int total = n_tiles_m * tiles_n;
    Cut8 cut = CUT ? plan_cut_upto(most_cut, total, ncu, K / kBlockK) : Cut8{total, 0, 1, 0};
    if (CUT) {                                               // the same for all blocks; the compiler does not see it through the divisions
        cut.n_full = __builtin_amdgcn_readfirstlane(cut.n_full);
        cut.n_tail = __builtin_amdgcn_readfirstlane(cut.n_tail);
        cut.parts = __builtin_amdgcn_readfirstlane(cut.parts);
        cut.per = __builtin_amdgcn_readfirstlane(cut.per);
    }
    const WalkRun run = walk_run(blockIdx.x, ncu, walk, cut.n_full + cut.n_tail * cut.parts);
    int item = run.item;
    const int end_item = run.end;
    if (item >= end_item) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
    const int all_blocks = K / kBlockK;

    constexpr int NB = EPI == EPI_SWIGLU ? NJ / 2 : NJ;
    struct Source { const uint8_t *a, *b0, *b1; uint32_t a_voff[MI], b_voff[NB]; };
    auto rsrc = [](const uint8_t* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, 0xFFFFFFFFu, 0x00027000); };
    auto describe = [&](int id, Item8& w, Source& src) {
        int lr, lc, ln = lane;
        asm volatile("" : "+v"(ln));                         // (opaque: not worth registers during the loop)
        rc_of_slot(ln, &lr, &lc);
        w.piece = -1;
        w.tail = 0;
        w.blocks = all_blocks;
        int first = 0;                                       // block of K
        if (CUT && id >= cut.n_full) {
            w.tail = (id - cut.n_full) % cut.n_tail;
            w.piece = (id - cut.n_full) / cut.n_tail;
            id = cut.n_full + w.tail;
            first = w.piece * cut.per;
            w.blocks = min(cut.per, all_blocks - first);
        }
        int tile_m, tile_n;
        tile_of_block(id, total, n_tiles_m, tiles_n, Strips{0, 0}, &tile_m, &tile_n);
        tile_m = __builtin_amdgcn_readfirstlane(tile_m);
        auto rec = [&](const int32_t* p) { return reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p))[tile_m]; };
        w.row0 = rec(m.row0);
        w.nrows = rec(m.nrows);
        w.expert = rec(m.expert);
        w.rel = rec(m.gather) ? m.rel + (size_t)tile_m * kRelPitch : nullptr;
        w.n0 = __builtin_amdgcn_readfirstlane(tile_n * OG::NOUT);
        auto weight = [&](int which) { return reinterpret_cast<const uint8_t*>(which == 0 ? tab.w1[w.expert] : which == 1 ? tab.w_up[w.expert] : tab.w_down[w.expert]) + (size_t)first * kBlockK; };
        src.b0 = weight(which0);
        src.b1 = EPI == EPI_SWIGLU ? weight(which1) : src.b0;
        src.a = A + (size_t)w.row0 * lda + (size_t)first * kBlockK;
        int a_row[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) a_row[i] = min((wave + 4 * i) * 16 + lr, w.nrows - 1);
        if (w.rel) {
            int u[MI];
#pragma unroll
            for (int i = 0; i < MI; ++i) u[i] = w.rel[a_row[i]];
#pragma unroll
            for (int i = 0; i < MI; ++i) a_row[i] = u[i];
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) src.a_voff[i] = (uint32_t)a_row[i] * (uint32_t)lda + (uint32_t)lc * 16u;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            // SwiGLU: gate rows of 64 columns, up rows of the same, gate rows of the next 64 ...; a lane's rows of the two have one offset
            static_assert(EPI != EPI_SWIGLU || NJ == 4, "");
            src.b_voff[i] = (uint32_t)min(w.n0 + (wave + 4 * i) * 16 + lr, N - 1) * (uint32_t)K + (uint32_t)lc * 16u;
        }
    };
    Item8 cur, next;
    Source src, src_next;
    int t_first = 0, t_last = 0;                             // the stage number at which `src` starts, and its last pair
    // Past the end of the last tile its last pair is fetched again (into stages nobody reads any more): the count of outstanding loads stays uniform
    auto pair_offset = [&](int t) { return min(t - t_first, t_last) * kKt; };
    auto issue_one = [&](int kb, int so0, int so1, int l) {  // load l of a pair: both halves of a line one after the other, A and B in turn
        const int it = l >> 1;
        const bool is_a = it < 2 * MI && (it & 1) == 0;
        const int i = it < 2 * MI ? it >> 1 : it - MI;
        unsigned char* to = lds + ((l & 1) ? so1 : so0) + (wave + 4 * i) * 1024 + (is_a ? 0 : TG::A_BYTES);
        // SwiGLU: 16-row block wave + 4 i holds up rows where r / (16 NJ) is odd
        const bool up = EPI == EPI_SWIGLU && (i & (NJ / 4));
        load_to_lds(rsrc(is_a ? src.a : up ? src.b1 : src.b0), to, is_a ? src.a_voff[i] : src.b_voff[EPI == EPI_SWIGLU ? i / 2 : i], kb + (l & 1) * kKt);
    };

    // A fragment is 16 rows x 64 bytes; lane: row lane % 16, chunk lane / 16 (the order of the sum is free)
    constexpr int NI = 2 * MI, NC = 2 * NJ;                  // fragments of a wave
    const int a_off = tile_off(wm * 32 * MI + (lane & 15), lane >> 4), b_off = TG::A_BYTES + tile_off(wn * 32 * NJ + (lane & 15), lane >> 4);
    i32x4 acc[NI][NC];
    // Read r of the NI + NC of a stage, in the order in which the products need them
    auto read = [&](i32x4 (&af)[NI], i32x4 (&bf)[NC], const unsigned char* st, int r) {
        if (r == 0) bf[0] = *reinterpret_cast<const i32x4*>(st + b_off);
        else if (r <= NI) af[r - 1] = *reinterpret_cast<const i32x4*>(st + a_off + (r - 1) * 1024);
        else bf[r - NI] = *reinterpret_cast<const i32x4*>(st + b_off + (r - NI) * 1024);
    };
    auto stage_products = [&](auto from_zero, const i32x4 (&af)[NI], const i32x4 (&bf)[NC], i32x4 (&an)[NI], i32x4 (&bn)[NC], const unsigned char* next_stage, auto n_loads, auto load) {
        constexpr int READS = NI + NC, L = decltype(n_loads)::value, M = NI * NC, EARLY = M * 5 / 8;   // the reads are done before the last products are
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[j], af[i], decltype(from_zero)::value ? i32x4{0, 0, 0, 0} : acc[i][j], 0, 0, 0);
                const int n = j * NI + i;                    // products before this one
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int l = n * L / M; l < (n + 1) * L / M; ++l) load(l);
#pragma unroll
                for (int r = n * READS / EARLY; r < (n + 1) * READS / EARLY; ++r)
                    if (r < READS) read(an, bn, next_stage, r);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    int so[TG::STAGES];
#pragma unroll
    for (int j = 0; j < TG::STAGES; ++j) so[j] = j * TG::STAGE;
    i32x4 a0[NI], a1[NI], b0[NC], b1[NC];                    // of even and odd stages
    describe(item, cur, src);
    t_last = 2 * cur.blocks - 2;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int l = 0; l < LOADS; ++l) issue_one(pair_offset(2 * q), so[2 * q], so[2 * q + 1], l);
    bool more = item + ncu < end_item;
    if (more) describe(item + ncu, next, src_next);
    __builtin_amdgcn_s_waitcnt(0x0F70 | ((P - 1) * LOADS & 15) | ((P - 1) * LOADS >> 4) << 14);   // vmcnt: pair (0, 1) is in LDS
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < NI + NC; ++r) read(a0, b0, lds + so[0], r);
    // One trip: a pair of stages, block kb of K.  SWITCH: the loads of this tile have all gone out, those of the next one follow.
    auto trip = [&](int kb, auto first, auto switches) {
        constexpr bool FIRST_TRIP = decltype(first)::value, SWITCH = decltype(switches)::value;
        const unsigned char *s1 = lds + so[1], *s2 = lds + so[2];
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);                  // lgkmcnt(0): this wave has read stage so[0], which is refilled below
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if ((SWITCH || (FIRST_TRIP && cur.blocks == 2)) && more) { src = src_next; t_first = 2 * cur.blocks; t_last = 2 * next.blocks - 2; }
        const int kt = 2 * kb, at = pair_offset(kt + 2 * P);
        stage_products(first, a0, b0, a1, b1, s1, std::integral_constant<int, FIRST>{}, [&](int l) { issue_one(at, so[2 * P], so[0], l); });
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (OPEN & 15) | (OPEN >> 4) << 14);   // the next pair is in LDS; lgkmcnt(0): this wave has read stage so[1]
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        stage_products(std::false_type{}, a1, b1, a0, b0, s2, std::integral_constant<int, LOADS - FIRST>{}, [&](int l) { issue_one(at, so[2 * P], so[0], FIRST + l); });
        __builtin_amdgcn_sched_barrier(0);
        const int t0 = so[0], t1 = so[1];
#pragma unroll
        for (int j = 0; j + 2 < TG::STAGES; ++j) so[j] = so[j + 2];
        so[2 * P - 1] = t0; so[2 * P] = t1;
    };
    while (true) {
        trip(0, std::true_type{}, std::false_type{});
        if (cur.blocks > 1) {                                // (a tile that another one follows has two at least)
            int kb = 1;
            for (; kb < cur.blocks - 2; ++kb) trip(kb, std::false_type{}, std::false_type{});
            if (cur.blocks > 2) {
                trip(kb, std::false_type{}, std::true_type{});
                ++kb;
            }
            trip(kb, std::false_type{}, std::false_type{});
        }
        asm volatile("s_nop 15\n\ts_nop 15");                // the last product has left the matrix core
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NC; ++j) asm volatile("" : "+a"(acc[i][j]));
        if (CUT && cur.piece >= 0) break;                    // the last item of its block: a round holds all pieces
        const Item8 done = cur;
        const bool had_next = more;
        if (more) {
            cur = next;
            t_first = 0;
            more = item + 2 * ncu < end_item;
        }
        const int col0 = __builtin_amdgcn_readfirstlane(done.n0 + wn * OG::NW);
        unsigned char* const stage = lds + so[2 * P];        // the only stage that no load is on its way to
        int ln = lane;
        asm volatile("" : "+v"(ln));
        if (col0 < N) {                                      // N is a multiple of 128: all columns of the wave or none
            constexpr int NT = OG::NW / 16;                  // 16-column tiles per wave
            const float* const cs0 = (EPI == EPI_PLAIN ? tab.s_down[done.expert] : tab.s1[done.expert]) + col0;
            const float* const cs1 = EPI == EPI_SWIGLU ? tab.s_up[done.expert] + col0 : cs0;
            f32x4 s0[NT], s1[NT];
            // the rows' scales: in registers, or where those are short in LDS behind the waves' regions
            constexpr bool IN_LDS = MI == 4;
            static_assert(!IN_LDS || TG::STAGE >= 4 * 4096 + 4 * 512, "");
            float rs[IN_LDS ? 1 : NI];
            float* const rs_lds = reinterpret_cast<float*>(stage + 4 * 4096 + wave * 512);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                s0[j] = *reinterpret_cast<const f32x4*>(cs0 + 16 * j + 4 * (ln >> 4));
                if (EPI == EPI_SWIGLU) s1[j] = *reinterpret_cast<const f32x4*>(cs1 + 16 * j + 4 * (ln >> 4));
            }
            if constexpr (IN_LDS) {
#pragma unroll
                for (int i = 0; i < 2; ++i) rs_lds[64 * i + ln] = row_scale(A, lda, K, done, wm * 128 + 64 * i + ln);
            } else {
#pragma unroll
                for (int i = 0; i < NI; ++i) rs[i] = row_scale(A, lda, K, done, wm * 32 * MI + 16 * i + (ln & 15));
            }
            auto factor = [&](int i) { return IN_LDS ? rs_lds[16 * i + (ln & 15)] : rs[IN_LDS ? 0 : i]; };
            auto value = [&](int i, int j, int e, float f) {
                const float a = (float)from_agpr_i(acc[i][j][e]) * s0[j][e] * f;
                return activation_fast<EPI>(a, EPI == EPI_SWIGLU ? (float)from_agpr_i(acc[i][(j + NJ) % NC][e]) * s1[j][e] * f : 0.f);
            };
            store_rows<NI, NT>(value, factor, ln, stage + wave * 4096, __builtin_amdgcn_make_buffer_rsrc(C + (size_t)__builtin_amdgcn_readfirstlane(done.row0) * ldc + (size_t)col0 * 2, 0, 0xFFFFFF00u, 0x00027000),
                               wm * 32 * MI, done, ldc);
        }
        if (!had_next) {
            __builtin_amdgcn_s_waitcnt(0x0070);              // no load may still target LDS when the block ends
            return;
        }
        item += ncu;
        if (more) describe(item + ncu, next, src_next);
    }
    if constexpr (CUT) {                                     // the raw sums, 16 bytes per lane and store
        __builtin_amdgcn_s_waitcnt(0x0070);                  // no load may still target LDS when the block ends
        constexpr int QUADS = TG::BM * TG::BN / 4;           // of a piece
        i32x4* const to = reinterpret_cast<i32x4*>(pieces) + ((size_t)cur.tail * cut.parts + cur.piece) * QUADS + tid;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                i32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = from_agpr_i(acc[i][j][e]);
                to[(i * NC + j) * 256] = v;
            }
    }
}

// Adds the pieces of the cut 256 x 256 tiles of the second GEMM: a block per tile and 16 x 64 of every wave's part
__global__ __launch_bounds__(256) void gemm_int8_sum_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTableI tab, int N, int K, char* __restrict__ C, int ldc, int tiles_n, int ncu,
                                                            int most_cut, const int* __restrict__ pieces) {
    constexpr int QUADS = 256 * 256 / 4;
    const int n_tiles_m = *m.n_tiles, total = n_tiles_m * tiles_n, tail = blockIdx.x / 16, unit = blockIdx.x % 16;
    const Cut8 cut = plan_cut_upto(most_cut, total, ncu, K / kBlockK);
    if (tail >= cut.n_tail) return;
    int tile_m, tile_n;
    tile_of_block(cut.n_full + tail, total, n_tiles_m, tiles_n, Strips{0, 0}, &tile_m, &tile_n);
    const int nrows = m.nrows[tile_m];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = (wave >> 1) * 128 + unit / 2 * 16 + (lane & 15), col = tile_n * 256 + (wave & 1) * 128 + unit % 2 * 64 + 4 * (lane >> 4);
    if (row >= nrows || col >= N) return;
    const i32x4* const from = reinterpret_cast<const i32x4*>(pieces) + (size_t)tail * cut.parts * QUADS + unit * 4 * 256 + threadIdx.x;
    i32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) v[g] = from[g * 256];
    for (int p = 1; p < cut.parts; ++p)
#pragma unroll
        for (int g = 0; g < 4; ++g) v[g] += from[(size_t)p * QUADS + g * 256];
    const size_t at = (size_t)m.row0[tile_m] + (m.gather[tile_m] ? m.rel[(size_t)tile_m * kRelPitch + row] : row);
    const float rs = *reinterpret_cast<const float*>(A + at * lda + K);
    const float* const cs = tab.s_down[m.expert[tile_m]] + col;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(cs + 16 * g);
        *reinterpret_cast<u32x2*>(C + at * ldc + (size_t)(col + 16 * g) * 2) =
            u32x2{pack_bf16((float)v[g][0] * s[0] * rs, (float)v[g][1] * s[1] * rs), pack_bf16((float)v[g][2] * s[2] * rs, (float)v[g][3] * s[3] * rs)};
    }
}

// ------------------------------------------------------------------------------------ few rows per expert
// A decode step reads every weight for a handful of rows: bound by memory.  A block takes 16 WV output columns and a tile of up to 16 MT rows over K or a piece of it; each of its WV
// waves takes 16 columns.  Rows, which all waves read, and weights, which no two share, go through a ring of D + 1 blocks of K in LDS, 8 rows of a whole 128-byte line per load,
// and from there to v_mfma_i32_16x16x64_i8 (lane: weight row lane % 16, 16 bytes of each half of a block's 128; the order of the sum is free).  One barrier per block of K.
//
// 64 columns a block (WV = 4) while such blocks are at most one per CU, else 128: 37 rows of 4096 -> 14336, SwiGLU, 224 blocks of 64 columns 24 to 31 us (117 MB, 3.8 to 4.8 TB/s), 224 of
// 128, each half of K, 31 and more often so; 403 rows of 2048 -> 1408, four experts, 352 blocks in two rounds 18.1, 176 of 128 columns 13.5.  Few blocks are cut along K, and the piece that
// arrives last adds all pieces (see last_piece): 14336 -> 4096, four pieces, 17 us (59 MB, 3.4 TB/s).  Rings as deep as LDS holds take the same time; weights and rows fetched straight
// to registers, 16 columns a block, 38 us instead of 29, as the rows come again for every 16 columns.
//
// The first GEMM's blocks work out their tile from the list of segments, if that is short and nothing is cut, and leave the map of tiles to the second: 4.7 us of a launch less.
// Pieces along K: as many as fill the chip's CUs with a block of 64 columns each, of at least four blocks of K
inline int stream_parts(int tiles, int N, int K) { return std::max(1, std::min(kStreamPieces / (tiles * (N / 64)), K / kBlockK / 4)); }
template <int EPI, int MT, int WV> struct StreamI {
    static constexpr int NF = EPI == EPI_SWIGLU ? 2 : 1;     // weight fragments per wave
    static constexpr int BM = 16 * MT;
    static constexpr int ROWS = BM * kBlockK, OWN = 16 * NF * kBlockK;         // bytes of a stage: rows, one wave's weights
    static constexpr int STAGE = ROWS + WV * OWN;
    static constexpr int D = (EPI == EPI_SWIGLU ? 16 : 32) / WV;
    static constexpr int PIECE = WV * NF * MT * 64;          // 16-byte units of a piece
    static constexpr int LOADERS = BM / 8 < WV ? BM / 8 : WV, ROW_LOADS = BM / 8 / LOADERS;   // waves that fetch the rows of a stage, and how many times 8 each
    static constexpr int LDS = (D + 1) * STAGE + 16;
};
template <int EPI, int MT, int WV>
__global__ __launch_bounds__(64 * WV, 2) void gemm_int8_stream_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTableI tab, int N, int K, char* __restrict__ C, int ldc,
                                                                      float* pieces, int max_tiles, int parts, SegList list) {
    using SG = StreamI<EPI, MT, WV>;
    constexpr int NF = SG::NF, D = SG::D, BM = SG::BM;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, quarter = lane >> 4;
    // Blocks go to the 8 XCDs in turn.  Those that read the same weights - the tiles of rows of one piece of one group of columns - are neighbours on one XCD.
    const int groups = N / (16 * WV), tile = blockIdx.x / 8 % max_tiles, unit = blockIdx.x / 8 / max_tiles * 8 + blockIdx.x % 8;
    const int group = unit % groups, part = unit / groups;
    if (part >= parts) return;
    int row0, nrows, ex;
    const int32_t* rel = nullptr;
    const int loader = wave % SG::LOADERS;
    int at_rows[SG::ROW_LOADS + MT];                         // rows of the tile that this lane fetches, and those whose sums it gets: where they are from row0 on
#pragma unroll
    for (int l = 0; l < SG::ROW_LOADS; ++l) at_rows[l] = 8 * (loader + l * SG::LOADERS) + (lane >> 3);
#pragma unroll
    for (int q = 0; q < MT; ++q) at_rows[SG::ROW_LOADS + q] = 16 * q + r;
    if (EPI != EPI_PLAIN && list.nseg > 0) {
        WaveLanes wl;
        const SmallMap sm = load_segments(list, BM, wl);
        if (blockIdx.x == 0) {                               // for the kernels behind this one, as the records below
            if (threadIdx.x == 0) *m.n_tiles = sm.n_tiles;
            for (int i = threadIdx.x; i < kMaxSplitTiles; i += 64 * WV) m.done[kMaxSplitTiles + i] = 0;
        }
        if (tile >= sm.n_tiles) return;
        const SmallTile st = small_tile(wl, sm, tile, BM);
        row0 = st.row0, nrows = st.nrows, ex = st.expert;
#pragma unroll
        for (int& v : at_rows) v = min(v, nrows - 1);
        segment_rows(wl, st, at_rows);
        if (group == 0 && wave == 0) {
            int all[1] = {lane};
            segment_rows(wl, st, all);
            if (lane == 0) {
                m.row0[tile] = row0;
                m.nrows[tile] = nrows;
                m.expert[tile] = ex;
                m.gather[tile] = st.gather;
            }
            if (st.gather && lane < nrows) m.rel[(size_t)tile * kRelPitch + lane] = all[0];
        }
    } else {
        if (tile >= *m.n_tiles) return;
        row0 = m.row0[tile], nrows = m.nrows[tile], ex = m.expert[tile];
        rel = m.gather[tile] ? m.rel + (size_t)tile * kRelPitch : nullptr;
#pragma unroll
        for (int& v : at_rows) v = min(v, nrows - 1);
        if (rel)
#pragma unroll
            for (int& v : at_rows) v = rel[v];
    }
    const int nb = K / kBlockK, kb0 = nb * part / parts, n = nb * (part + 1) / parts - kb0;   // n >= 1 (see stream_parts)
    auto rsrc = [](const void* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000); };
    const void *const w0 = EPI == EPI_PLAIN ? tab.w_down[ex] : tab.w1[ex], *const w1 = EPI == EPI_SWIGLU ? tab.w_up[ex] : w0, *const rows = A + (size_t)row0 * lda;
    // With fewer than 8 WV rows several waves fetch the same ones (to the same place: the count of outstanding loads is every wave's)
    uint32_t a_off[SG::ROW_LOADS];
#pragma unroll
    for (int l = 0; l < SG::ROW_LOADS; ++l) a_off[l] = (uint32_t)at_rows[l] * (uint32_t)lda + (((lane & 7) ^ stream_swizzle((8 * (loader + l * SG::LOADERS) + (lane >> 3)) & 15)) << 4);
    // past the end nothing is fetched (zeros, from descriptors without bytes): the count of outstanding loads stays uniform.  (The compiler forms the size in a vector register; a
    // descriptor that is not scalar costs a loop per load.)
    auto bytes_at = [&](int i) { return (uint32_t)__builtin_amdgcn_readfirstlane(i < n ? -1 : 0); };
    auto load_rows = [&](int i, int stage) {
        const uint32_t bytes = bytes_at(i);
#pragma unroll
        for (int l = 0; l < SG::ROW_LOADS; ++l) load_to_lds(rsrc(rows, bytes), lds + stage * SG::STAGE + (loader + l * SG::LOADERS) * 1024, a_off[l], (kb0 + i) * kBlockK);
    };
    // a load: 8 of the wave's 16 columns, whole lines
    uint32_t w_off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w_off[h] = (uint32_t)(group * 16 * WV + wave * 16 + 8 * h + (lane >> 3)) * (uint32_t)K + (((lane & 7) ^ stream_swizzle(8 * h + (lane >> 3))) << 4);
    auto load_weights = [&](int i, int stage) {
        const int at = (kb0 + i) * kBlockK;
        const uint32_t bytes = bytes_at(i);
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) load_to_lds(rsrc(j == 0 ? w0 : w1, bytes), lds + stage * SG::STAGE + SG::ROWS + wave * SG::OWN + (2 * j + h) * 1024, w_off[h], at);
    };
    // the scales go out first: lane: rows 16 q + lane % 16, columns 4 (lane / 16) ... + 3 of the wave's 16
    const int col = group * 16 * WV + wave * 16 + 4 * quarter;
    float rs[MT];
    f32x4 cs[NF];
#pragma unroll
    for (int q = 0; q < MT; ++q) rs[q] = *reinterpret_cast<const float*>(A + ((size_t)row0 + at_rows[SG::ROW_LOADS + q]) * lda + K);
    cs[0] = *reinterpret_cast<const f32x4*>((EPI == EPI_PLAIN ? tab.s_down[ex] : tab.s1[ex]) + col);
    if (NF == 2) cs[NF - 1] = *reinterpret_cast<const f32x4*>(tab.s_up[ex] + col);
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_rows(d, d);
        load_weights(d, d);
    }
    i32x4 acc[NF][MT];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = i32x4{0, 0, 0, 0};
    const int frag = r * kBlockK + ((quarter ^ stream_swizzle(r)) << 4);
    int stage = 0;
    for (int i = 0; i < n; ++i) {
        // what was issued for blocks i + 1 .. i + D - 1 may be outstanding; lgkmcnt(0): this wave has read the stage that is refilled below
        constexpr int OPEN = (D - 1) * (2 * NF + SG::ROW_LOADS);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (OPEN & 15) | (OPEN >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        load_rows(i + D, stage == 0 ? D : stage - 1);
        load_weights(i + D, stage == 0 ? D : stage - 1);
        const unsigned char *const st = lds + stage * SG::STAGE, *const own = st + SG::ROWS + wave * SG::OWN;
        i32x4 w[NF][2];
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) w[j][h] = *reinterpret_cast<const i32x4*>(own + (frag ^ (64 * h)) + j * 2048);
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const i32x4 a = *reinterpret_cast<const i32x4*>(st + (frag ^ (64 * h)) + q * 2048);
#pragma unroll
                for (int j = 0; j < NF; ++j) acc[j][q] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j][h], a, acc[j][q], 0, 0, 0);
            }
        stage = stage == D ? 0 : stage + 1;
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                      // no load may still target LDS
    __builtin_amdgcn_s_barrier();
    if (parts > 1) {
        const size_t id = ((size_t)tile * groups + group) * parts;
        const __amdgpu_buffer_rsrc_t dst = pieces_rsrc(pieces + id * SG::PIECE * 4, (uint32_t)parts * SG::PIECE * 16);
        const int own = wave * NF * MT * 64 + lane, used = (nrows + 15) / 16;
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int q = 0; q < MT; ++q)
                if (q < used) store_piece(dst, part * SG::PIECE + own + (j * MT + q) * 64, __builtin_bit_cast(f32x4, acc[j][q]));
        if (!last_piece(m.done + tile * groups + group, parts, reinterpret_cast<int*>(lds + (D + 1) * SG::STAGE))) return;
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int q = 0; q < MT; ++q) acc[j][q] = i32x4{0, 0, 0, 0};
        for (int p0 = 0; p0 < parts; p0 += 4) {              // four pieces are requested before the first is added (past the last one that again, not added)
            f32x4 v[4][NF][MT];
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < MT; ++q) v[p][j][q] = load_piece(dst, min(p0 + p, parts - 1) * SG::PIECE + own + (j * MT + min(q, used - 1)) * 64);
#pragma unroll
            for (int p = 0; p < 4; ++p)
                if (p0 + p < parts)
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int q = 0; q < MT; ++q) acc[j][q] += __builtin_bit_cast(i32x4, v[p][j][q]);
        }
    }
#pragma unroll
    for (int q = 0; q < MT; ++q) {
        const int row = 16 * q + r;
        if (row >= nrows) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = (float)acc[0][q][e] * cs[0][e] * rs[q];
            v[e] = activation_fast<EPI>(a, NF == 2 ? (float)acc[NF - 1][q][e] * cs[NF - 1][e] * rs[q] : 0.f);
        }
        const size_t at = (size_t)row0 + at_rows[SG::ROW_LOADS + q];
        *reinterpret_cast<u32x2*>(C + at * ldc + (size_t)col * 2) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
}

template <int EPI, int MT, int WV>
int launch_stream_mt(const uint8_t* A, const TileMap& m, const ExpertTableI& tab, int N, int K, void* C, int ldc, int tiles, int parts, float* pieces, const SegList& list, hipStream_t st) {
    static LdsLimit limit;
    if (const int rc = raise_lds_limit(limit, reinterpret_cast<const void*>(&gemm_int8_stream_kernel<EPI, MT, WV>), StreamI<EPI, MT, WV>::LDS)) return rc;
    hipLaunchKernelGGL((gemm_int8_stream_kernel<EPI, MT, WV>), dim3((N / (16 * WV) * parts + 7) / 8 * 8 * tiles), dim3(64 * WV), (StreamI<EPI, MT, WV>::LDS), st, A, (int)int8_row_bytes(K), m,
                       tab, N, K, reinterpret_cast<char*>(C), ldc, pieces, tiles, parts, list);
    MOE_LAUNCH_CHECK("gemm_int8_stream_kernel");
    return MOE_OK;
}
template <int EPI>
int launch_stream(int mt, const uint8_t* A, const TileMap& m, const ExpertTableI& tab, int N, int K, void* C, int ldc, int tiles, float* pieces, const SegList& list, hipStream_t st) {
    const int parts = stream_parts(tiles, N, K);             // 1 where the blocks have 128 columns
#define MOE_STREAM(MT, WV) launch_stream_mt<EPI, MT, WV>(A, m, tab, N, K, C, ldc, tiles, parts, pieces, list, st)
    if (tiles * (N / 64) <= kStreamPieces) return mt == 1 ? MOE_STREAM(1, 4) : mt == 2 ? MOE_STREAM(2, 4) : MOE_STREAM(4, 4);
    return mt == 1 ? MOE_STREAM(1, 8) : mt == 2 ? MOE_STREAM(2, 8) : MOE_STREAM(4, 8);
#undef MOE_STREAM
}

// P > 2: no walk
template <int EPI, int MI, int NJ, int P>
int launch_tile(const uint8_t* A, const TileMap& m, const ExpertTableI& tab, int which0, int which1, int N, int K, void* C, int ldc, int R, int nseg, int n_used, int* pieces, hipStream_t st) {
    using TG = Geom8<MI, NJ, P>;
    constexpr bool CUT = EPI == EPI_PLAIN && MI == 4;
    static LdsLimit limit;
    if (const int rc = raise_lds_limit(limit, reinterpret_cast<const void*>(&gemm_int8_kernel<EPI, MI, NJ, P, CUT>), TG::LDS)) return rc;
    const int lda = (int)int8_row_bytes(K), tiles_n = (N + Out8<EPI, NJ>::NOUT - 1) / Out8<EPI, NJ>::NOUT, ncu = round_size() * TG::PER_CU;
    const int walk = K < 2 * kBlockK || P > 2 ? 1 : std::max(1, (int)(210.0 / (5.0 + 0.55 * (K / kKt))));
    // the tile count is known on the device only: the most tiles cut over every count that n_used runs of rows which share no tile can give
    int most_cut = 0;
    if (CUT && pieces)
        for (int t = (R + TG::BM - 1) / TG::BM, hi = (int)((R + (int64_t)n_used * (TG::BM - 1)) / TG::BM); t <= hi; ++t)
            most_cut = std::max(most_cut, plan_cut(t * tiles_n, ncu, K / kBlockK).n_tail);
    hipLaunchKernelGGL((gemm_int8_kernel<EPI, MI, NJ, P, CUT>), dim3(walk_blocks(max_tiles_of(R, TG::BM, nseg) * tiles_n + (CUT ? ncu : 0), walk, ncu)), dim3(256), TG::LDS, st, A, lda, m, tab,
                       which0, which1, N, K, reinterpret_cast<char*>(C), ldc, tiles_n, ncu, walk, most_cut, pieces);
    MOE_LAUNCH_CHECK("gemm_int8_kernel");
    if (most_cut > 0) {
        hipLaunchKernelGGL(gemm_int8_sum_kernel, dim3(most_cut * 16), dim3(256), 0, st, A, lda, m, tab, N, K, reinterpret_cast<char*>(C), ldc, tiles_n, ncu, most_cut, pieces);
        MOE_LAUNCH_CHECK("gemm_int8_sum_kernel");
    }
    return MOE_OK;
}
// bm: rows per tile (64: SwiGLU); deep: 128 x 128 tiles of one block per CU, with a ring of four pairs of stages
template <int EPI>
int launch_int8(int bm, const uint8_t* A, const TileMap& m, const ExpertTableI& tab, int which0, int which1, int N, int K, void* C, int ldc, int R, int nseg, int n_used, bool deep, int* pieces, hipStream_t st) {
    if (bm == 256) return launch_tile<EPI, 4, 4, 2>(A, m, tab, which0, which1, N, K, C, ldc, R, nseg, n_used, pieces, st);
    if constexpr (EPI == EPI_SWIGLU) {
        if (bm == 64) return launch_tile<EPI, 1, 4, 3>(A, m, tab, which0, which1, N, K, C, ldc, R, nseg, n_used, pieces, st);
        return launch_tile<EPI, 2, 4, 2>(A, m, tab, which0, which1, N, K, C, ldc, R, nseg, n_used, pieces, st);
    } else {
        if constexpr (EPI == EPI_PLAIN)
            if (deep) return launch_tile<EPI, 2, 2, 4>(A, m, tab, which0, which1, N, K, C, ldc, R, nseg, n_used, pieces, st);
        return launch_tile<EPI, 2, 2, 2>(A, m, tab, which0, which1, N, K, C, ldc, R, nseg, n_used, pieces, st);
    }
}

// Sums of 127 * 128 * K stay in 32 bits up to this; weights, and the 256 rows of a tile in every array, are addressed by 32-bit byte offsets
constexpr int kMostK = 130944;
bool sizes_ok(int H, int F) {
    return H > 0 && F > 0 && H % kBlockK == 0 && F % kBlockK == 0 && H <= kMostK && F <= kMostK && (size_t)H * F <= 0xFFFFFFFFull;
}
size_t widest_row(int H, int F) { return 2 * std::max((size_t)H, (size_t)F); }
// The weights are streamed for few rows whatever K is, as nothing that grows with it stays in LDS.  One expert, in tiles of 128 and 256 rows and streamed: 4096 -> 32896 -> 4096
// SwiGLU, 1 row 169 and 127 us, 64 rows 171 and 142; 2048 -> 130944 -> 2048 319 and 170, 328 and 201; 40960 -> 8192 -> 40960 367 and 208, 60 rows 406 and 224.  Four of 512 -> 33024 -> 512
// SiLU, 60 rows 82 and 50; 400 rows, where the estimate of the choice is off, 89 and 102.
Plan8 plan_int8(int R, int n_used, int nseg, int H, int F, int act, bool gather) { return plan_ffn8(R, n_used, nseg, H, F, act, gather, kMostK); }

}  // namespace

extern "C" int moe_selfcheck_int8_plan(int32_t R, int32_t n_used, int32_t nseg, int32_t H, int32_t F, int32_t act, int32_t* plan5) {
    if (R < 1 || n_used < 1 || n_used > R || nseg < n_used || nseg > kMaxSeg || !sizes_ok(H, F) || act < 0 || act > 2 || !plan5)
        return moe_set_error(MOE_EINVAL, "moe_selfcheck_int8_plan: bad argument");
    const Plan8 p = plan_int8(R, n_used, nseg, H, F, act, true);
    plan5[0] = p.mt; plan5[1] = p.bm[0]; plan5[2] = p.bm[1]; plan5[3] = plan5[4] = 0;
    if (!p.mt) return MOE_OK;
    const int tiles = (R + n_used * (p.bm[0] - 1)) / p.bm[0];
    for (int g = 0; g < 2; ++g) {
        const int N = g == 0 ? F : H, K = g == 0 ? H : F, blocks = K / kBlockK, parts = stream_parts(tiles, N, K);
        if (parts > 1 && (tiles * (N / 64) * parts > kStreamPieces || tiles * (N / 64) > kMaxSplitTiles)) return moe_set_error(MOE_EINTERNAL, "the pieces do not fit");
        for (int i = 0; i < parts; ++i)
            if (blocks * (i + 1) / parts <= blocks * i / parts) return moe_set_error(MOE_EINTERNAL, "a piece without blocks");
        plan5[3 + g] = parts;
    }
    return MOE_OK;
}

extern "C" int moe_quantize_int8(const void* x, int32_t T, int32_t H, int32_t dtype, void* rows, void* stream) {
    if (T != 0 && (!x || !rows)) return moe_set_error(MOE_EINVAL, "moe_quantize_int8: NULL argument");
    if (T < 0 || H <= 0) return moe_set_error(MOE_EINVAL, "moe_quantize_int8: T >= 0 and H > 0 required");
    if (dtype != MOE_F32 && dtype != MOE_BF16) return moe_set_error(MOE_EDTYPE, "moe_quantize_int8: unknown dtype %d", dtype);
    if (H % kBlockK != 0 || H > kMostK) return moe_set_error(MOE_ESHAPE, "moe_quantize_int8: H must be a multiple of 128 and at most %d", kMostK);
    if (!aligned16(x) || !aligned16(rows)) return moe_set_error(MOE_EALIGN, "moe_quantize_int8: x and rows must be 16-byte aligned");
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return dtype == MOE_BF16 ? launch_quantize<MOE_BF16>(x, T, H, reinterpret_cast<uint8_t*>(rows), st) : launch_quantize<MOE_F32>(x, T, H, reinterpret_cast<uint8_t*>(rows), st);
}

extern "C" size_t moe_ffn_int8_workspace_bytes(int32_t R_max, int32_t H, int32_t F, int32_t act) {
    if (R_max < 0 || !sizes_ok(H, F) || act < 0 || act > 2) return 0;
    const size_t bytes = tilemap_bytes(R_max) + align256((size_t)R_max * F * 2) + align256((size_t)R_max * int8_row_bytes(F));
    // whatever R_max is: a share of fewer rows may be run another way
    return bytes + std::max((size_t)kStreamPieces * StreamI<EPI_SWIGLU, 4, 4>::PIECE * 16, may_cut(F) ? (size_t)kCutPieces * 256 * 256 * sizeof(int) : 0);
}

extern "C" int moe_expert_ffn_int8(const void* recv, int32_t R, const int32_t* seg_offset, const int32_t* seg_expert, int32_t nseg,
                                   const moe_expert_wi8* experts, int32_t n_local, int32_t H, int32_t F, int32_t act, void* out,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if ((R != 0 && (!recv || !out)) || !seg_offset || (nseg != 0 && !seg_expert) || !experts || !workspace) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_int8: NULL argument");
    if (R < 0 || nseg < 0 || H <= 0 || F <= 0) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_int8: negative size");
    if (act < 0 || act > 2) return moe_set_error(MOE_EDTYPE, "moe_expert_ffn_int8: unknown act %d", act);
    if (n_local < 1 || n_local > MOE_MAX_LOCAL || nseg > kMaxSeg)
        return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_int8: need 1 <= n_local <= %d and nseg <= %d", MOE_MAX_LOCAL, kMaxSeg);
    if (!sizes_ok(H, F)) return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_int8: H and F must be multiples of 128 and at most %d, weight matrices below 4 GiB", kMostK);
    if (!aligned16(recv) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return moe_set_error(MOE_EALIGN, "moe_expert_ffn_int8: recv/out need 16-byte, workspace 256-byte alignment");
    if (workspace_bytes < moe_ffn_int8_workspace_bytes(R, H, F, act))
        return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_int8: workspace too small (%zu < %zu)", workspace_bytes, moe_ffn_int8_workspace_bytes(R, H, F, act));
    ExpertTableI tab;
    for (int e = 0; e < n_local; ++e) {
        const moe_expert_wi8& w = experts[e];
        if (!w.w1 || !w.w_down || !w.s1 || !w.s_down || (act == MOE_ACT_SWIGLU && (!w.w_up || !w.s_up)))
            return moe_set_error(MOE_EINVAL, "moe_expert_ffn_int8: expert %d has a NULL weight or scale", e);
        if (!aligned16(w.w1) || !aligned16(w.w_down) || !aligned16(w.w_up) || !aligned16(w.s1) || !aligned16(w.s_up) || !aligned16(w.s_down))
            return moe_set_error(MOE_EALIGN, "moe_expert_ffn_int8: expert %d weights and scales must be 16-byte aligned", e);
        tab.w1[e] = w.w1; tab.w_up[e] = w.w_up; tab.w_down[e] = w.w_down;
        tab.s1[e] = w.s1; tab.s_up[e] = w.s_up; tab.s_down[e] = w.s_down;
    }
    if (R == 0 || nseg == 0) return MOE_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    char* const h = reinterpret_cast<char*>(workspace) + tilemap_bytes(R);
    uint8_t* const hq = reinterpret_cast<uint8_t*>(h + align256((size_t)R * F * 2));
    // gathered tiles address their rows by 32-bit byte offsets from the tile's first row, in every array
    const int gather = (size_t)R * widest_row(H, F) <= 0xFFFFFF00ull ? 1 : 0;
    const int n_used = std::min(gather ? std::min(n_local, nseg) : nseg, R);   // runs of rows that share no tile
    const Plan8 p = plan_int8(R, n_used, nseg, H, F, act, gather);
    MapJobs jobs = {};
    jobs.job[0] = MapJob{p.bm[0], max_tiles_of(R, p.bm[0], nseg), tilemap_at(workspace, R)};
    jobs.job[1] = p.bm[1] == p.bm[0] ? jobs.job[0] : MapJob{p.bm[1], max_tiles_of(R, p.bm[1], nseg), tilemap_at(workspace, R, 1, jobs.job[0].max_tiles)};
    jobs.done = tilemap_at(workspace, R, 0, max_tiles_for(R) - 2).rel;
    jobs.job[0].m.done = jobs.done;
    jobs.job[1].m.done = jobs.done + kMaxSplitTiles;
    const int n_maps = p.bm[1] == p.bm[0] ? 1 : 2;
    const int tiles = (R + n_used * (p.bm[0] - 1)) / p.bm[0];   // at most, of shares that stream the weights
    const bool by_list = p.mt > 0 && nseg <= kSmallMapSegs && stream_parts(tiles, F, H) == 1;
    const SegList list = {seg_offset, seg_expert, by_list ? nseg : 0, R, n_local, gather, jobs.job[0].max_tiles};
    if (!by_list) {
        const int blocks = std::min(64, (R / std::min(p.bm[0], p.bm[1]) + std::min(nseg, n_local) + 3) / 4);
        if (nseg <= kSmallMapSegs) hipLaunchKernelGGL(tilemap_small_kernel<false>, dim3(blocks, n_maps), dim3(256), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
        else hipLaunchKernelGGL(tilemap_kernel, dim3(n_maps), dim3(kMapThreads), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
        MOE_LAUNCH_CHECK("tilemap_kernel");
    }
    const TileMap &m = jobs.job[0].m, &m2 = jobs.job[1].m;
    const uint8_t* const in = reinterpret_cast<const uint8_t*>(recv);
    float* const pieces = reinterpret_cast<float*>(reinterpret_cast<char*>(hq) + align256((size_t)R * int8_row_bytes(F)));
    int rc;
    if (p.mt) {
        if (act == MOE_ACT_SWIGLU) rc = launch_stream<EPI_SWIGLU>(p.mt, in, m, tab, F, H, h, F * 2, tiles, pieces, list, st);
        else if (act == MOE_ACT_GELU_MLP) rc = launch_stream<EPI_GELU>(p.mt, in, m, tab, F, H, h, F * 2, tiles, pieces, list, st);
        else rc = launch_stream<EPI_SILU>(p.mt, in, m, tab, F, H, h, F * 2, tiles, pieces, list, st);
    } else {
        if (act == MOE_ACT_SWIGLU) rc = launch_int8<EPI_SWIGLU>(p.bm[0], in, m, tab, 0, 1, F, H, h, F * 2, R, nseg, n_used, false, nullptr, st);
        else if (act == MOE_ACT_GELU_MLP) rc = launch_int8<EPI_GELU>(p.bm[0], in, m, tab, 0, 0, F, H, h, F * 2, R, nseg, n_used, false, nullptr, st);
        else rc = launch_int8<EPI_SILU>(p.bm[0], in, m, tab, 0, 0, F, H, h, F * 2, R, nseg, n_used, false, nullptr, st);
    }
    if (rc != MOE_OK) return rc;
    // (rows outside every segment hold whatever was there: nobody reads them)
    if ((rc = launch_quantize<MOE_BF16>(h, R, F, hq, st)) != MOE_OK) return rc;
    if (p.mt) return launch_stream<EPI_PLAIN>(p.mt, hq, m2, tab, H, F, out, H * 2, tiles, pieces, list, st);
    return launch_int8<EPI_PLAIN>(p.bm[1], hq, m2, tab, 2, 2, H, F, out, H * 2, R, nseg, n_used, p.deep, may_cut(F) ? reinterpret_cast<int*>(pieces) : nullptr, st);
}
