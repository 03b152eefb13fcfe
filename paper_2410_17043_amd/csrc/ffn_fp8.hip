// Expert FFN on 8-bit rows and weights (e4m3 with a power-of-two scale per 128 elements), a ragged grouped GEMM pair.
//
//   GEMM1  h = act(recv . W1^T [, recv . Wu^T]), quantised per 128 columns into packed rows
//   GEMM2  out = h . Wd^T, bf16
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies e4m3 operands with a power-of-two scale per row and 32 elements of K in the instruction
// itself, so the scales of a block of 128 cost no arithmetic.  The map of tiles is that of the bf16 kernels (ffn_tiles.h).
//
// Roundings: sums in fp32; h to e4m3 (the layer's format, the only rounding to fewer bits between the GEMMs); out to bf16.  The matrix cores' e4m3 products are
// themselves off by 1.5e-5 of a sum of 2048 normal products (measured outside the library, against 64 bits, on chains of single instructions of 32x32x64, 32x32x16 and 16x16x32,
// with the sum in the accumulator and added in fp32: the same).
// So an element of h that lies that near to the middle of two e4m3 values, or a block whose largest element lies that near to a power of two times 448, can
// be rounded to the neighbour: of the tiles, out is 0.0018 to 0.0029 off a form that rounds the exact h, where rounding out to bf16 alone is 0.0017.  Few rows, which stream the weights,
// are where single elements weigh most and where the matrix cores have time: there the first product's operands are widened to bf16, and out is 0.0017 off.
#include "ffn_tiles8.h"
#include <type_traits>

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ExpertTable8 {
    const void *w1[MOE_MAX_LOCAL], *w_up[MOE_MAX_LOCAL], *w_down[MOE_MAX_LOCAL];
    const uint8_t *s1[MOE_MAX_LOCAL], *s_up[MOE_MAX_LOCAL], *s_down[MOE_MAX_LOCAL];
};

// Stores of a wave's part of a tile.  acc[i][j][e]: row 32 i + lane % 32, column 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4.  Four
// neighbouring columns of a row are one 8- or 4-byte piece; 32 rows at a time cross LDS (`region`, this wave's own) and
// leave as whole 128- (bf16) or 64-byte (e4m3) runs.  Region: rows of 16-byte chunks, chunk c of row r at slot c ^ (r / rows per 256 bytes), and in
// rows 16-31 the two halves of every chunk change places, which spreads a write of 32 rows over all 64 banks.
template <int MI, int NJ>
__device__ __forceinline__ void store_bf16(const f32x16 (&acc)[MI][NJ], int lane, unsigned char* region, __amdgpu_buffer_rsrc_t dst, int first_row, const Item8& t, int ldc) {
    const int r = lane & 31, half = lane >> 5;
    unsigned char* const wr = region + r * 128 + ((half ^ (r >> 4)) << 3);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        uint32_t off[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) off[it] = row_offset(t, first_row + 32 * i + 8 * it + (lane >> 3), ldc) + (lane & 7) * 16;
#pragma unroll
        for (int p = 0; p < NJ / 2; ++p) {                   // 64 columns
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& a = acc[i][2 * p + j];
                    const u32x2 q = {pack_bf16(from_agpr(a[4 * g]), from_agpr(a[4 * g + 1])), pack_bf16(from_agpr(a[4 * g + 2]), from_agpr(a[4 * g + 3]))};
                    *reinterpret_cast<u32x2*>(wr + (((4 * j + g) ^ ((r >> 1) & 7)) << 4)) = q;
                }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int rr = 8 * it + (lane >> 3);
                u32x4 q = *reinterpret_cast<const u32x4*>(region + rr * 128 + (((lane & 7) ^ ((rr >> 1) & 7)) << 4));
                if (it >= 2) q = u32x4{q[2], q[3], q[0], q[1]};
                __builtin_amdgcn_raw_buffer_store_b128(q, dst, off[it], p * 128, 0);
            }
        }
    }
}

// The same for an activation: quantised per 128 columns, which are one wave's (NW = 128) or those of the two waves of a row of waves (NW = 64),
// who then tell each other the largest element of every row through LDS (`most`, 4 x 32 words).
template <int EPI, int MI, int NJ>
__device__ __forceinline__ void store_fp8(const f32x16 (&acc)[MI][NJ], int lane, int wave, unsigned char* region, uint32_t* most, __amdgpu_buffer_rsrc_t dst, int first_row,
                                          const Item8& t, int ldc, int scale_col, bool live) {
    constexpr int NT = Out8<EPI, NJ>::NW / 32;               // 32-column tiles per wave
    constexpr bool SHARED = NT == 2;
    const int r = lane & 31, half = lane >> 5;
    const int wr = r * 64 + ((half ^ (r >> 4 << 1)) << 2);   // (an offset: a pointer that passes through an integer is no LDS pointer any more)
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        float v[NT][16];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                v[j][e] = activation_fast<EPI>(from_agpr(acc[i][j][e]), EPI == EPI_SWIGLU ? from_agpr(acc[i][(j + NJ / 2) % NJ][e]) : 0.f);
                m = max(m, abs_bits(v[j][e]));
            }
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if (SHARED) {
            asm volatile("" ::: "memory");
            if (half == 0) most[(i & 1) * 128 + wave * 32 + r] = m;
            lds_barrier();
            m = max(m, most[(i & 1) * 128 + (wave ^ 1) * 32 + r]);
        }
        const bool bad = fp8_block_is_nan(m);
        const uint32_t b = bad ? 127u : fp8_scale_byte(m);
        const float inv = fp8_inverse_scale(b);
        uint32_t off[2];
#pragma unroll
        for (int it = 0; it < 2; ++it) off[it] = row_offset(t, first_row + 32 * i + 16 * it + (lane >> 2), ldc) + (lane & 3) * 16;
#pragma unroll
        for (int p = 0; p < NT / 2; ++p) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float (&a)[16] = v[2 * p + j];
                    const uint32_t q = bad ? 0x7f7f7f7fu : fp8_pack4(a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3], inv);
                    *reinterpret_cast<uint32_t*>(region + (wr ^ ((g & 1) << 3)) + (((2 * j + (g >> 1)) ^ ((r >> 2) & 3)) << 4)) = q;
                }
            asm volatile("" ::: "memory");
            if (live)
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const int rr = 16 * it + (lane >> 2);
                    u32x4 q = *reinterpret_cast<const u32x4*>(region + rr * 64 + (((lane & 3) ^ ((rr >> 2) & 3)) << 4));
                    if (it == 1) q = u32x4{q[2], q[3], q[0], q[1]};
                    __builtin_amdgcn_raw_buffer_store_b128(q, dst, off[it], p * 64, 0);
                }
        }
        if (live && half == 0 && (!SHARED || (wave & 1) == 0))
            __builtin_amdgcn_raw_buffer_store_b8((unsigned char)b, dst, row_offset(t, first_row + 32 * i + r, ldc) , scale_col, 0);
    }
}

// C = epilogue(A . B^T) for one tile of 64 MI rows and 64 NJ weight rows.  SwiGLU: the weight rows are, per wave column wn (16 NJ output
// columns), 16 NJ rows of W1 followed by the 16 NJ rows of Wu for the same columns, so that a lane has the gate and the up product of a column.
//
// Pipeline, as in the bf16 kernels (the bytes per product are half, so are the cycles: a k-tile of 64 bytes is 1024 cycles of products per wave in
// both): five stages of a k-tile, loads straight to LDS in pairs of k-tiles, spread between the products, fragments read a k-tile ahead, one barrier
// per k-tile; the pipeline runs on across the tiles that a block walks through.  A pair of k-tiles is 128 elements, one block of scales.
// Those of the rows are words of four blocks in a register per 32 rows, loaded four blocks ahead and shifted to the block at hand; those of the weights,
// the same for a whole wave, are one byte per lane, taken by lane number.
// 256 x 256: 20571 rows of 4096 -> 14336 SwiGLU 1.95 ms (2.48 PFLOP/s), back 0.93 (2.60): bound by power, matrix cores 64-73 % busy at 1.7 GHz.  Smaller tiles: by bytes in
// flight and LDS reads; 403 rows of 2048 -> 1408 SwiGLU for four experts 16 us, back 10.5.
template <int EPI, int MI, int NJ, int P, bool CUT>
__global__ __launch_bounds__(256, (Geom8<MI, NJ, P>::PER_CU)) void gemm_fp8_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTable8 tab, int which0, int which1, int N, int K,
                                                          char* __restrict__ C, int ldc, int tiles_n, int ncu, int walk, int most_cut, float* pieces) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    using TG = Geom8<MI, NJ, P>;
    using OG = Out8<EPI, NJ>;
    constexpr int LOADS = 2 * (MI + NJ), FIRST = MI + NJ;    // loads per pair of k-tiles and wave; those in the first half of a trip
    constexpr int OPEN = (P - 2) * LOADS + FIRST;            // loads that may be outstanding in the middle of a trip: those of pairs that are needed later
    static_assert(OPEN < 64 && P >= 2, "");
    auto word = [](const int32_t* p) { return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p)); };
    const int n_tiles_m = word(m.n_tiles);
    const int total = n_tiles_m * tiles_n;
    Cut8 cut = CUT ? plan_cut_upto(most_cut, total, ncu, K / FP8_BLOCK) : Cut8{total, 0, 1, 0};
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
    const int all_blocks = K / FP8_BLOCK;

    struct Source { const uint8_t *a, *b0, *b1, *s0, *s1; uint32_t a_voff[MI], b_voff[NJ], s_voff[MI]; };
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
        const int ex = rec(m.expert);
        w.rel = rec(m.gather) ? m.rel + (size_t)tile_m * kRelPitch : nullptr;
        w.n0 = __builtin_amdgcn_readfirstlane(tile_n * OG::NOUT);
        auto weight = [&](int which) { return reinterpret_cast<const uint8_t*>(which == 0 ? tab.w1[ex] : which == 1 ? tab.w_up[ex] : tab.w_down[ex]) + (size_t)first * FP8_BLOCK; };
        const size_t scale_row = (size_t)(min(w.n0 + wn * OG::NW, N - FP8_BLOCK) / FP8_BLOCK) * all_blocks + first;
        auto scales = [&](int which) { return (which == 0 ? tab.s1[ex] : which == 1 ? tab.s_up[ex] : tab.s_down[ex]) + scale_row; };
        src.b0 = weight(which0);
        src.s0 = scales(which0);
        src.b1 = EPI == EPI_SWIGLU ? weight(which1) : src.b0;
        src.s1 = EPI == EPI_SWIGLU ? scales(which1) : src.s0;
        src.a = A + (size_t)w.row0 * lda + (size_t)first * FP8_BLOCK;
        int a_row[MI], s_row[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            a_row[i] = min((wave + 4 * i) * 16 + lr, w.nrows - 1);
            s_row[i] = min(wm * 32 * MI + 32 * i + (ln & 31), w.nrows - 1);
        }
        if (w.rel) {
            int u[MI], v[MI];
#pragma unroll
            for (int i = 0; i < MI; ++i) { u[i] = w.rel[a_row[i]]; v[i] = w.rel[s_row[i]]; }
#pragma unroll
            for (int i = 0; i < MI; ++i) { a_row[i] = u[i]; s_row[i] = v[i]; }
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            src.a_voff[i] = (uint32_t)a_row[i] * (uint32_t)lda + (uint32_t)lc * 16u;
            src.s_voff[i] = (uint32_t)s_row[i] * (uint32_t)lda + (uint32_t)(K - first * (FP8_BLOCK - 1));
        }
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const int r = (wave + 4 * i) * 16 + lr;          // tile row this lane fetches
            int col = w.n0 + r;
            if (EPI == EPI_SWIGLU) {
                constexpr int WB = 32 * NJ;                  // weight rows per wave column, the first half gate, the second up
                col = w.n0 + r / WB * (WB / 2) + r % (WB / 2);
            }
            src.b_voff[i] = (uint32_t)min(col, N - 1) * (uint32_t)K + (uint32_t)lc * 16u;
        }
    };
    Item8 cur, next;
    Source src, src_next;
    int t_first = 0, t_last = 0;                             // the k-tile number at which `src` starts, and its last pair
    // Past the end of the last tile its last pair is fetched again (into stages nobody reads any more): the count of outstanding loads stays uniform
    auto pair_offset = [&](int t) { return min(t - t_first, t_last) * kKt; };
    auto issue_one = [&](int kb, int so0, int so1, int l) {  // load l of a pair: both halves of a line one after the other, A and B in turn
        const int it = l >> 1;
        const bool is_a = it < 2 * MI && (it & 1) == 0;
        const int i = it < 2 * MI ? it >> 1 : it - MI;
        unsigned char* to = lds + ((l & 1) ? so1 : so0) + (wave + 4 * i) * 1024 + (is_a ? 0 : TG::A_BYTES);
        // SwiGLU: 16-row block wave + 4 i holds up rows where r / (16 NJ) is odd
        const bool up = EPI == EPI_SWIGLU && (i & (NJ / 4));
        load_to_lds(rsrc(is_a ? src.a : up ? src.b1 : src.b0), to, is_a ? src.a_voff[i] : src.b_voff[i], kb + (l & 1) * kKt);
    };

    struct Scales { uint32_t rows[MI]; uint32_t w0, w1; };
    auto load_scales = [&](const Source& s, int blocks, int g, Scales& to) {
#pragma unroll
        for (int i = 0; i < MI; ++i) to.rows[i] = __builtin_amdgcn_raw_buffer_load_b32(rsrc(s.a), s.s_voff[i], g * 4, 0);
        const int at = min(g * 4 + (lane & 3), blocks - 1);
        to.w0 = __builtin_amdgcn_raw_buffer_load_b8(rsrc(s.s0), at, 0, 0);
        if (EPI == EPI_SWIGLU) to.w1 = __builtin_amdgcn_raw_buffer_load_b8(rsrc(s.s1), at, 0, 0);
    };

    // A fragment is 32 rows x 64 bytes; lane: row lane % 32, bytes 32 (lane / 32) ..., two chunks
    const int a_off = tile_off(wm * 32 * MI + (lane & 31), (lane >> 5) * 2), b_off = TG::A_BYTES + tile_off(wn * 32 * NJ + (lane & 31), (lane >> 5) * 2);
    f32x16 acc[MI][NJ];
    struct Frag { u32x4 lo, hi; };
    auto whole = [](const Frag& f) {
        typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
        const u32x8 v = __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return *reinterpret_cast<const i32x8*>(&v);
    };
    // Read r of the 2 (MI + NJ) of a k-tile, in the order in which the products need them
    auto read = [&](Frag (&af)[MI], Frag (&bf)[NJ], const unsigned char* st, int r) {
        const int f = r >> 1;
        Frag& to = f == 0 ? bf[0] : f <= MI ? af[f - 1] : bf[f - MI];
        const int off = f == 0 ? b_off : f <= MI ? a_off + (f - 1) * 2048 : b_off + (f - MI) * 2048;
        if (r & 1) to.hi = *reinterpret_cast<const u32x4*>(st + (off ^ 16));
        else to.lo = *reinterpret_cast<const u32x4*>(st + off);
    };
    auto k_tile = [&](auto from_zero, const Frag (&af)[MI], const Frag (&bf)[NJ], Frag (&an)[MI], Frag (&bn)[NJ], const unsigned char* next_stage, const int (&sa)[MI], int sb0, int sb1,
                      auto n_loads, auto load) {
        constexpr int READS = 2 * (MI + NJ), L = decltype(n_loads)::value, M = MI * NJ, EARLY = M * 5 / 8;   // the reads are done before the last products are
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                f32x16 zero;
#pragma unroll
                for (int e = 0; e < 16; ++e) zero[e] = 0.f;
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(bf[j]), whole(af[i]), decltype(from_zero)::value ? zero : acc[i][j], 0, 0,
                                                                           0, EPI == EPI_SWIGLU && j >= NJ / 2 ? sb1 : sb0, 0, sa[i]);
                const int n = j * MI + i;                    // products before this one
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
    Frag a0[MI], a1[MI], b0[NJ], b1[NJ];                     // of even and odd k-tiles
    Scales sc, sc_next;
    describe(item, cur, src);
    t_last = 2 * cur.blocks - 2;
    load_scales(src, cur.blocks, 0, sc);
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
    for (int r = 0; r < 2 * (MI + NJ); ++r) read(a0, b0, lds + so[0], r);
    // One trip: a pair of k-tiles, block kb of the scales.  SWITCH: the loads of this tile have all gone out, those of the next one follow.
    auto trip = [&](int kb, auto first, auto switches) {
        constexpr bool FIRST_TRIP = decltype(first)::value, SWITCH = decltype(switches)::value;
        const unsigned char *s1 = lds + so[1], *s2 = lds + so[2];
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);                  // lgkmcnt(0): this wave has read stage so[0], which is refilled below
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if ((kb & 3) == 0) {                                 // the scales of the next four blocks, or of the next tile's first
            if (kb + 4 < cur.blocks) load_scales(src, cur.blocks, kb / 4 + 1, sc_next);
            else if (more) load_scales(src_next, next.blocks, 0, sc_next);
        }
        if ((SWITCH || (FIRST_TRIP && cur.blocks == 2)) && more) { src = src_next; t_first = 2 * cur.blocks; t_last = 2 * next.blocks - 2; }
        int sa[MI];
        const int sh = (kb & 3) * 8;
#pragma unroll
        for (int i = 0; i < MI; ++i) sa[i] = (int)(sc.rows[i] >> sh);
        const int sb0 = __builtin_amdgcn_readlane(sc.w0, kb & 3), sb1 = EPI == EPI_SWIGLU ? __builtin_amdgcn_readlane(sc.w1, kb & 3) : sb0;
        const int kt = 2 * kb, at = pair_offset(kt + 2 * P);
        k_tile(first, a0, b0, a1, b1, s1, sa, sb0, sb1, std::integral_constant<int, FIRST>{}, [&](int l) { issue_one(at, so[2 * P], so[0], l); });
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (OPEN & 15) | (OPEN >> 4) << 14);   // the next pair is in LDS; lgkmcnt(0): this wave has read stage so[1]
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        k_tile(std::false_type{}, a1, b1, a0, b0, s2, sa, sb0, sb1, std::integral_constant<int, LOADS - FIRST>{}, [&](int l) { issue_one(at, so[2 * P], so[0], FIRST + l); });
        __builtin_amdgcn_sched_barrier(0);
        if ((kb & 3) == 3 || kb == cur.blocks - 1) sc = sc_next;
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
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
        if (CUT && cur.piece >= 0) break;                    // the last item of its block: a round holds all pieces
        const Item8 done = cur;
        const bool had_next = more;
        if (more) {
            cur = next;
            t_first = 0;
            more = item + 2 * ncu < end_item;
        }
        const int col0 = __builtin_amdgcn_readfirstlane(done.n0 + wn * OG::NW);
        const bool live = col0 < N;                          // N is a multiple of 128: all columns of the wave or none
        unsigned char* const stage = lds + so[2 * P];        // the only stage that no load is on its way to
        int ln = lane;
        asm volatile("" : "+v"(ln));
        char* const row0 = C + (size_t)__builtin_amdgcn_readfirstlane(done.row0) * ldc;
        if (EPI == EPI_PLAIN) {
            if (live)
                store_bf16<MI, NJ>(acc, ln, stage + wave * 4096, __builtin_amdgcn_make_buffer_rsrc(row0 + (size_t)col0 * 2, 0, 0xFFFFFF00u, 0x00027000), wm * 32 * MI, done, ldc);
        } else {
            store_fp8<EPI, MI, NJ>(acc, ln, wave, stage + wave * 2048, reinterpret_cast<uint32_t*>(stage + 8192),
                                   __builtin_amdgcn_make_buffer_rsrc(row0 + col0, 0, 0xFFFFFF00u, 0x00027000), wm * 32 * MI, done, ldc, N + col0 / FP8_BLOCK - col0, live);
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
        f32x4* const to = reinterpret_cast<f32x4*>(pieces) + ((size_t)cur.tail * cut.parts + cur.piece) * QUADS + tid;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = from_agpr(acc[i][j][4 * g + e]);
                    to[((i * NJ + j) * 4 + g) * 256] = v;
                }
    }
}

// Adds the pieces of the cut 256 x 256 tiles in their order: a block per tile and 32 x 32 of every wave's part
__global__ __launch_bounds__(256) void gemm_fp8_sum_kernel(TileMap m, int N, int K, char* __restrict__ C, int ldc, int tiles_n, int ncu, int most_cut, const float* __restrict__ pieces) {
    constexpr int QUADS = 256 * 256 / 4;
    const int n_tiles_m = *m.n_tiles, total = n_tiles_m * tiles_n, tail = blockIdx.x / 16, unit = blockIdx.x % 16;
    const Cut8 cut = plan_cut_upto(most_cut, total, ncu, K / FP8_BLOCK);
    if (tail >= cut.n_tail) return;
    int tile_m, tile_n;
    tile_of_block(cut.n_full + tail, total, n_tiles_m, tiles_n, Strips{0, 0}, &tile_m, &tile_n);
    const int nrows = m.nrows[tile_m];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = (wave >> 1) * 128 + unit / 4 * 32 + (lane & 31), col = tile_n * 256 + (wave & 1) * 128 + unit % 4 * 32 + 4 * (lane >> 5);
    if (row >= nrows || col >= N) return;
    const f32x4* const from = reinterpret_cast<const f32x4*>(pieces) + (size_t)tail * cut.parts * QUADS + unit * 4 * 256 + threadIdx.x;
    f32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) v[g] = from[g * 256];
    for (int p = 1; p < cut.parts; ++p)
#pragma unroll
        for (int g = 0; g < 4; ++g) v[g] += from[(size_t)p * QUADS + g * 256];
    const size_t at = (size_t)m.row0[tile_m] + (m.gather[tile_m] ? m.rel[(size_t)tile_m * kRelPitch + row] : row);
#pragma unroll
    for (int g = 0; g < 4; ++g) *reinterpret_cast<u32x2*>(C + at * ldc + (size_t)(col + 8 * g) * 2) = u32x2{pack_bf16(v[g][0], v[g][1]), pack_bf16(v[g][2], v[g][3])};
}

// ------------------------------------------------------------------------------------ few rows per expert
// A decode step reads every weight for a handful of rows: bound by memory.  A block takes 128 output columns (the columns that are quantised together) and a
// tile of up to 16 MT rows over K or a piece of it; each of its 8 waves takes 16 columns.  Rows, which all waves read, and weights, which no two share, go through a ring of
// D + 1 blocks of K in LDS, 8 rows of a whole 128-byte line per load, and from there to the matrix cores (lane: weight row lane % 16, 16 bytes of each half of a
// block's 128; the order of the sum is free): in the second GEMM as they are, by v_mfma_scale_f32_16x16x128_f8f6f4; in the first, whose sums are rounded to 8 bits, widened to bf16 with
// their scales and by v_mfma_f32_16x16x32_bf16, in which products are exact (403 rows of four experts of 2048 -> 1408 26.3 -> 27.2 us, 128 of 4096 -> 14336 66 -> 71, 37 55.4 -> 55.3; scales applied to a
// block's sum instead 28.2, 72.4, 54.9).  The scales of rows and weights are fetched to LDS once.  One barrier per block of K.  Few column blocks are cut along K, and the piece that arrives
// last adds all pieces in their order (see last_piece).  37 rows of 4096 -> 14336 SwiGLU 30.4 us, back 20.3: 117 and 59 MB of weights at up to 4.6 TB/s inside the loop, the rest start and the sum of two
// and eight pieces.  Weights straight to registers, 16 rows of half a line per load: 33 and 22; for 100 rows of eight experts of 2048 -> 5632 the share 80 instead of 66; deeper rings gave nothing (when each load's descriptor was in vector registers and cost a loop).
constexpr int kStreamWaves = 8, kStreamBlocks = 256;         // waves of a block; blocks of K that the scales in LDS have room for
template <int EPI, int MT> struct Stream8 {
    static constexpr int NF = EPI == EPI_SWIGLU ? 2 : 1;     // weight fragments per wave
    static constexpr int D = EPI == EPI_SWIGLU ? 2 : 4;
    static constexpr int BM = 16 * MT;
    static constexpr int ROWS = BM * FP8_BLOCK, OWN = 16 * NF * FP8_BLOCK;     // bytes of a stage: rows, one wave's weights
    static constexpr int STAGE = ROWS + kStreamWaves * OWN;
    static constexpr int PIECE = kStreamWaves * NF * MT * 64;          // 16-byte units of a piece
    static constexpr int LOADERS = BM / 8;                             // waves that it takes to fetch the rows of a stage, 8 each
    static int lds(int nb) { return (D + 1) * STAGE + (BM + 2) * ((nb + 15) & ~15) + kStreamWaves * BM * 4; }
};
// 32 e4m3 numbers with their scale as bf16, which holds them exactly (down to 2^-133)
struct Bf16x32 { bf16x8 g[4]; };
__device__ __forceinline__ Bf16x32 widen(const u32x4& lo, const u32x4& hi, uint32_t scale_byte) {
    const float scale = __uint_as_float(scale_byte << 23);
    Bf16x32 v;
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t q = (g < 2 ? lo : hi)[2 * (g & 1) + i];
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, true);
            v.g[g][4 * i] = a[0]; v.g[g][4 * i + 1] = a[1]; v.g[g][4 * i + 2] = b[0]; v.g[g][4 * i + 3] = b[1];
        }
    return v;
}

template <int EPI, int MT>
__global__ __launch_bounds__(64 * kStreamWaves, 2) void gemm_fp8_stream_kernel(const uint8_t* __restrict__ A, int lda, TileMap m, ExpertTable8 tab, int N, int K,
                                                                               char* __restrict__ C, int ldc, float* pieces, int max_tiles, int parts) {
    using SG = Stream8<EPI, MT>;
    constexpr int NF = SG::NF, D = SG::D, BM = SG::BM;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, quarter = lane >> 4;
    // Blocks go to the 8 XCDs in turn.  Those that read the same weights - the tiles of rows of one piece of one group of columns - are neighbours on one XCD.
    const int groups = N / 128, tile = blockIdx.x / 8 % max_tiles, unit = blockIdx.x / 8 / max_tiles * 8 + blockIdx.x % 8;
    const int group = unit % groups, part = unit / groups;
    if (part >= parts || tile >= *m.n_tiles) return;
    const int row0 = m.row0[tile], nrows = m.nrows[tile], ex = m.expert[tile];
    const int32_t* rel = m.gather[tile] ? m.rel + (size_t)tile * kRelPitch : nullptr;
    const int nb = K / FP8_BLOCK, kb0 = nb * part / parts, n = nb * (part + 1) / parts - kb0;   // n >= 1 (see stream_pieces)
    const int strip = (nb + 15) & ~15;                       // scale bytes per row, in whole chunks (the padding of packed rows has room for them)
    unsigned char* const row_scales = lds + (D + 1) * SG::STAGE;
    unsigned char* const w_scales = row_scales + BM * strip;
    uint32_t* const most = reinterpret_cast<uint32_t*>(w_scales + 2 * strip);
    auto rsrc = [](const void* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000); };
    const void *const w0 = EPI == EPI_PLAIN ? tab.w_down[ex] : tab.w1[ex], *const w1 = EPI == EPI_SWIGLU ? tab.w_up[ex] : w0, *const rows = A + (size_t)row0 * lda;
    auto row_at = [&](int q) { const int c = min(q, nrows - 1); return (uint32_t)(rel ? rel[c] : c) * (uint32_t)lda; };
    // row of a stage that this lane fetches.  With fewer than 64 rows several waves fetch the same ones (to the same place: the count of outstanding loads is
    // every wave's)
    const int loader = wave % SG::LOADERS, my_row = 8 * loader + (lane >> 3);
    const uint32_t a_off = row_at(my_row) + (((lane & 7) ^ stream_swizzle(my_row & 15)) << 4);
    // past the end nothing is fetched (zeros, from descriptors without bytes): the count of outstanding loads stays uniform.  (The compiler forms the size in a vector register; a
    // descriptor that is not scalar costs a loop per load.)
    auto bytes_at = [&](int i) { return (uint32_t)__builtin_amdgcn_readfirstlane(i < n ? -1 : 0); };
    auto load_rows = [&](int i, int stage) {
        load_to_lds(rsrc(rows, bytes_at(i)), lds + stage * SG::STAGE + loader * 1024, a_off, (kb0 + i) * FP8_BLOCK);
    };
    // a load: 8 of the wave's 16 columns, whole lines
    uint32_t w_off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w_off[h] = (uint32_t)(group * 128 + wave * 16 + 8 * h + (lane >> 3)) * (uint32_t)K + (((lane & 7) ^ stream_swizzle(8 * h + (lane >> 3))) << 4);
    auto load_weights = [&](int i, int stage) {
        const int at = (kb0 + i) * FP8_BLOCK;
        const uint32_t bytes = bytes_at(i);
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) load_to_lds(rsrc(j == 0 ? w0 : w1, bytes), lds + stage * SG::STAGE + SG::ROWS + wave * SG::OWN + (2 * j + h) * 1024, w_off[h], at);
    };
    // The scales go out first and to LDS behind the loads of the first blocks: one round trip for both
    constexpr int SCALE_LOADS = BM * (kStreamBlocks / 16) / (64 * kStreamWaves) > 0 ? BM * (kStreamBlocks / 16) / (64 * kStreamWaves) : 1;
    static_assert(2 * kStreamBlocks <= 64 * kStreamWaves, "a scale byte of the weights per thread");
    u32x4 of_rows[SCALE_LOADS];
    uint8_t of_weights = 0;
#pragma unroll
    for (int u = 0; u < SCALE_LOADS; ++u) {
        const int i = threadIdx.x + u * 64 * kStreamWaves, q = i / (strip / 16), c = i % (strip / 16);
        if (q < BM) of_rows[u] = *reinterpret_cast<const u32x4*>(A + (size_t)row0 * lda + row_at(q) + K + c * 16);
    }
    const bool up = (int)threadIdx.x >= nb;
    if ((int)threadIdx.x < NF * nb)
        of_weights = (EPI == EPI_PLAIN ? tab.s_down[ex] : up ? tab.s_up[ex] : tab.s1[ex])[(size_t)group * nb + threadIdx.x - (up ? nb : 0)];
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_rows(d, d);
        load_weights(d, d);
    }
#pragma unroll
    for (int u = 0; u < SCALE_LOADS; ++u) {
        const int i = threadIdx.x + u * 64 * kStreamWaves, q = i / (strip / 16), c = i % (strip / 16);
        if (q < BM) *reinterpret_cast<u32x4*>(row_scales + q * strip + c * 16) = of_rows[u];
    }
    if ((int)threadIdx.x < NF * nb) w_scales[threadIdx.x + (up ? strip - nb : 0)] = of_weights;
    auto whole = [](const u32x4& lo, const u32x4& hi) {
        typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
        const u32x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return *reinterpret_cast<const i32x8*>(&v);
    };
    f32x4 acc[NF][MT];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int frag = r * FP8_BLOCK + ((quarter ^ stream_swizzle(r)) << 4);
    int stage = 0;
    for (int i = 0; i < n; ++i) {
        // what was issued for blocks i + 1 .. i + D - 1 may be outstanding; lgkmcnt(0): this wave has read the stage that is refilled below
        constexpr int OPEN = (D - 1) * (2 * NF + 1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (OPEN & 15) | (OPEN >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        load_rows(i + D, stage == 0 ? D : stage - 1);
        load_weights(i + D, stage == 0 ? D : stage - 1);
        const unsigned char *const st = lds + stage * SG::STAGE, *const own = st + SG::ROWS + wave * SG::OWN;
        const int kb = kb0 + i;
        auto row_lo = [&](int q) { return *reinterpret_cast<const u32x4*>(st + frag + q * 2048); };
        auto row_hi = [&](int q) { return *reinterpret_cast<const u32x4*>(st + (frag ^ 64) + q * 2048); };
        auto w_lo = [&](int j) { return *reinterpret_cast<const u32x4*>(own + frag + j * 2048); };
        auto w_hi = [&](int j) { return *reinterpret_cast<const u32x4*>(own + (frag ^ 64) + j * 2048); };
        if constexpr (EPI == EPI_PLAIN) {
            const i32x8 w = whole(w_lo(0), w_hi(0));
            const int sw = w_scales[kb];
#pragma unroll
            for (int q = 0; q < MT; ++q)
                acc[0][q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, whole(row_lo(q), row_hi(q)), acc[0][q], 0, 0, 0, sw, 0, row_scales[(16 * q + r) * strip + kb]);
        } else {
            Bf16x32 w[NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) w[j] = widen(w_lo(j), w_hi(j), w_scales[j * strip + kb]);
#pragma unroll
            for (int q = 0; q < MT; ++q) {
                const Bf16x32 a = widen(row_lo(q), row_hi(q), row_scales[(16 * q + r) * strip + kb]);
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int j = 0; j < NF; ++j) acc[j][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j].g[g], a.g[g], acc[j][q], 0, 0, 0);
            }
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
                if (q < used) store_piece(dst, part * SG::PIECE + own + (j * MT + q) * 64, acc[j][q]);
        if (!last_piece(m.done + tile * groups + group, parts, reinterpret_cast<int*>(most))) return;
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int q = 0; q < MT; ++q) acc[j][q] = f32x4{0.f, 0.f, 0.f, 0.f};
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
                        for (int q = 0; q < MT; ++q) acc[j][q] += v[p][j][q];
        }
        __syncthreads();                                     // `most` is free again
    }
    // lane: row 16 q + lane % 16, columns 4 (lane / 16) ... + 3 of the wave's 16
    const int col = group * 128 + wave * 16 + 4 * quarter;
    if (EPI == EPI_PLAIN) {
#pragma unroll
        for (int q = 0; q < MT; ++q) {
            const int row = 16 * q + r;
            if (row >= nrows) continue;
            const size_t at = (size_t)row0 + (rel ? rel[row] : row);
            *reinterpret_cast<u32x2*>(C + at * ldc + (size_t)col * 2) = u32x2{pack_bf16(acc[0][q][0], acc[0][q][1]), pack_bf16(acc[0][q][2], acc[0][q][3])};
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < MT; ++q) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[0][q][e] = activation_fast<EPI>(acc[0][q][e], acc[NF - 1][q][e]);
            top = max(top, abs_bits(acc[0][q][e]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        if (quarter == 0) most[wave * BM + 16 * q + r] = top;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < MT; ++q) {
        const int row = 16 * q + r;
        if (row >= nrows) continue;
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < kStreamWaves; ++v) top = max(top, most[v * BM + row]);
        const bool bad = fp8_block_is_nan(top);
        const uint32_t b = bad ? 127u : fp8_scale_byte(top);
        char* const out = C + ((size_t)row0 + (rel ? rel[row] : row)) * ldc;
        *reinterpret_cast<uint32_t*>(out + col) = bad ? 0x7f7f7f7fu : fp8_pack4(acc[0][q][0], acc[0][q][1], acc[0][q][2], acc[0][q][3], fp8_inverse_scale(b));
        if (wave == 0 && quarter == 0) out[N + group] = (char)b;
    }
}

template <int EPI, int MT>
int launch_stream_mt(const void* A, const TileMap& m, const ExpertTable8& tab, int N, int K, void* C, int ldc, int tiles, float* pieces, hipStream_t st) {
    const int bytes = Stream8<EPI, MT>::lds(K / FP8_BLOCK), parts = stream_pieces(tiles, N, K);
    static LdsLimit limit;
    if (const int rc = raise_lds_limit(limit, reinterpret_cast<const void*>(&gemm_fp8_stream_kernel<EPI, MT>), Stream8<EPI, MT>::lds(kStreamBlocks))) return rc;
    hipLaunchKernelGGL((gemm_fp8_stream_kernel<EPI, MT>), dim3((N / 128 * parts + 7) / 8 * 8 * tiles), dim3(64 * kStreamWaves), bytes, st, reinterpret_cast<const uint8_t*>(A),
                       (int)fp8_row_bytes(K), m, tab, N, K, reinterpret_cast<char*>(C), ldc, pieces, tiles, parts);
    MOE_LAUNCH_CHECK("gemm_fp8_stream_kernel");
    return MOE_OK;
}
template <int EPI>
int launch_stream(int mt, const void* A, const TileMap& m, const ExpertTable8& tab, int N, int K, void* C, int ldc, int tiles, float* pieces, hipStream_t st) {
#define MOE_STREAM(MT) launch_stream_mt<EPI, MT>(A, m, tab, N, K, C, ldc, tiles, pieces, st)
    return mt == 1 ? MOE_STREAM(1) : mt == 2 ? MOE_STREAM(2) : MOE_STREAM(4);
#undef MOE_STREAM
}

// P > 2: no walk
template <int EPI, int MI, int NJ, int P>
int launch_tile(const void* A, const TileMap& m, const ExpertTable8& tab, int which0, int which1, int N, int K, void* C, int ldc, int R, int nseg, int n_used, float* pieces, hipStream_t st) {
    using TG = Geom8<MI, NJ, P>;
    constexpr bool CUT = EPI == EPI_PLAIN && MI == 4;
    static LdsLimit limit;
    if (const int rc = raise_lds_limit(limit, reinterpret_cast<const void*>(&gemm_fp8_kernel<EPI, MI, NJ, P, CUT>), TG::LDS)) return rc;
    const int tiles_n = (N + Out8<EPI, NJ>::NOUT - 1) / Out8<EPI, NJ>::NOUT, ncu = round_size() * TG::PER_CU;
    const int walk = K < 2 * FP8_BLOCK || P > 2 ? 1 : std::max(1, (int)(210.0 / (5.0 + 0.55 * (K / kKt))));
    // the tile count is known on the device only: the most tiles cut over every count that n_used runs of rows which share no tile can give
    int most_cut = 0;
    if (CUT && pieces)
        for (int t = (R + TG::BM - 1) / TG::BM, hi = (int)((R + (int64_t)n_used * (TG::BM - 1)) / TG::BM); t <= hi; ++t)
            most_cut = std::max(most_cut, plan_cut(t * tiles_n, ncu, K / FP8_BLOCK).n_tail);
    hipLaunchKernelGGL((gemm_fp8_kernel<EPI, MI, NJ, P, CUT>), dim3(walk_blocks(max_tiles_of(R, TG::BM, nseg) * tiles_n + (CUT ? ncu : 0), walk, ncu)), dim3(256), TG::LDS, st,
                       reinterpret_cast<const uint8_t*>(A), (int)fp8_row_bytes(K), m, tab, which0, which1, N, K, reinterpret_cast<char*>(C), ldc, tiles_n, ncu, walk, most_cut, pieces);
    MOE_LAUNCH_CHECK("gemm_fp8_kernel");
    if (most_cut > 0) {
        hipLaunchKernelGGL(gemm_fp8_sum_kernel, dim3(most_cut * 16), dim3(256), 0, st, m, N, K, reinterpret_cast<char*>(C), ldc, tiles_n, ncu, most_cut, pieces);
        MOE_LAUNCH_CHECK("gemm_fp8_sum_kernel");
    }
    return MOE_OK;
}
// bm: rows per tile (64: SwiGLU); deep: 128 x 128 tiles of one block per CU, with a ring of four pairs of k-tiles
template <int EPI>
int launch_fp8(int bm, const void* A, const TileMap& m, const ExpertTable8& tab, int which0, int which1, int N, int K, void* C, int ldc, int R, int nseg, int n_used, bool deep, float* pieces, hipStream_t st) {
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

Plan8 plan_fp8(int R, int n_used, int nseg, int H, int F, int act, bool gather) { return plan_ffn8(R, n_used, nseg, H, F, act, gather, kStreamBlocks * FP8_BLOCK); }

// weights, and the 256 rows of a tile in every array, are addressed by 32-bit byte offsets
bool sizes_ok(int H, int F) {
    return H > 0 && F > 0 && H % FP8_BLOCK == 0 && F % FP8_BLOCK == 0 && (size_t)H * F <= 0xFFFFFFFFull &&
           256 * std::max<size_t>({fp8_row_bytes(H), fp8_row_bytes(F), (size_t)H * 2}) <= 0xFFFFFF00ull;
}

}  // namespace

extern "C" int moe_selfcheck_fp8_plan(int32_t R, int32_t n_used, int32_t nseg, int32_t H, int32_t F, int32_t act, int32_t ncu, int32_t* plan5) {
    if (R < 1 || n_used < 1 || n_used > R || nseg < n_used || nseg > kMaxSeg || !sizes_ok(H, F) || act < 0 || act > 2 || ncu < 1 || ncu > kCutPieces || !plan5)
        return moe_set_error(MOE_EINVAL, "moe_selfcheck_fp8_plan: bad argument");
    for (const bool gather : {false, true}) {
        const Plan8 q = plan_fp8(R, n_used, nseg, H, F, act, gather);
        if (free_records(R, nseg, q.bm[0], q.bm[1]) < 0 || (q.mt > 0 && !gather)) return moe_set_error(MOE_EINTERNAL, "the tile maps do not fit");
    }
    const Plan8 p = plan_fp8(R, n_used, nseg, H, F, act, true);
    plan5[0] = p.mt; plan5[1] = p.bm[0]; plan5[2] = p.bm[1]; plan5[3] = p.deep; plan5[4] = 1;
    if (p.mt) {
        const int tiles = (R + n_used * (p.bm[0] - 1)) / p.bm[0];
        for (int g = 0; g < 2; ++g) {
            const int N = g == 0 ? F : H, K = g == 0 ? H : F, blocks = K / FP8_BLOCK, parts = stream_pieces(tiles, N, K);
            if (parts > 1 && (tiles * (N / 128) * parts > kStreamPieces || tiles * (N / 128) > kMaxSplitTiles)) return moe_set_error(MOE_EINTERNAL, "the pieces do not fit");
            for (int i = 0; i < parts; ++i)
                if (blocks * (i + 1) / parts <= blocks * i / parts) return moe_set_error(MOE_EINTERNAL, "a piece without blocks");
            if (blocks > kStreamBlocks || p.mt > 4) return moe_set_error(MOE_EINTERNAL, "the scales do not fit");
            plan5[4] = parts;
        }
        return MOE_OK;
    }
    if (p.bm[1] != 256) return MOE_OK;
    const int blocks = F / FP8_BLOCK, tiles_n = (H + 255) / 256;
    for (int t = (R + 255) / 256; t <= (R + n_used * 255) / 256; ++t) {
        const Cut8 c = plan_cut(t * tiles_n, ncu, blocks);
        if (c.n_full + c.n_tail != t * tiles_n || c.n_full % ncu * c.n_tail != 0) return moe_set_error(MOE_EINTERNAL, "%d tiles are lost", t * tiles_n);
        if (c.parts > 1 && (!may_cut(F) || c.n_tail * c.parts > ncu || c.per % 4 != 0 || c.per * (c.parts - 1) >= blocks || c.per * c.parts < blocks))
            return moe_set_error(MOE_EINTERNAL, "pieces of %d tiles", t * tiles_n);
        plan5[4] = std::max(plan5[4], c.parts);
    }
    return MOE_OK;
}

extern "C" int moe_selfcheck_fp8_records(int32_t R, int32_t nseg, int32_t bm0, int32_t bm1) {
    if (R < 1 || nseg < 1 || nseg > kMaxSeg || bm0 < 1 || bm0 > kRelPitch || bm1 < 1 || bm1 > kRelPitch) return -(1 << 30);
    return free_records(R, nseg, bm0, bm1);
}

extern "C" size_t moe_ffn_fp8_workspace_bytes(int32_t R_max, int32_t H, int32_t F, int32_t act) {
    if (R_max < 0 || !sizes_ok(H, F) || act < 0 || act > 2) return 0;
    size_t bytes = tilemap_bytes(R_max) + align256((size_t)R_max * fp8_row_bytes(F)) + 256;
    // whatever R_max is: a share of fewer rows may be run another way
    return bytes + std::max((size_t)kStreamPieces * Stream8<EPI_SWIGLU, 4>::PIECE * 16, may_cut(F) ? (size_t)kCutPieces * 256 * 256 * sizeof(float) : 0);
}

extern "C" int moe_expert_ffn_fp8(const void* recv, int32_t R, const int32_t* seg_offset, const int32_t* seg_expert, int32_t nseg,
                                  const moe_expert_w8* experts, int32_t n_local, int32_t H, int32_t F, int32_t act, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if ((R != 0 && (!recv || !out)) || !seg_offset || (nseg != 0 && !seg_expert) || !experts || !workspace) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_fp8: NULL argument");
    if (R < 0 || nseg < 0 || H <= 0 || F <= 0) return moe_set_error(MOE_EINVAL, "moe_expert_ffn_fp8: negative size");
    if (act < 0 || act > 2) return moe_set_error(MOE_EDTYPE, "moe_expert_ffn_fp8: unknown act %d", act);
    if (n_local < 1 || n_local > MOE_MAX_LOCAL || nseg > kMaxSeg)
        return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_fp8: need 1 <= n_local <= %d and nseg <= %d", MOE_MAX_LOCAL, kMaxSeg);
    if (!sizes_ok(H, F)) return moe_set_error(MOE_ESHAPE, "moe_expert_ffn_fp8: H and F must be multiples of 128, weight matrices and 256 rows of every array below 4 GiB");
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
    // gathered tiles address their rows by 32-bit byte offsets from the tile's first row, in every array
    const int gather = (size_t)R * std::max<size_t>({fp8_row_bytes(H), fp8_row_bytes(F), (size_t)H * 2}) <= 0xFFFFFF00ull ? 1 : 0;
    const int n_used = std::min(gather ? std::min(n_local, nseg) : nseg, R);   // runs of rows that share no tile
    const Plan8 p = plan_fp8(R, n_used, nseg, H, F, act, gather);
    MapJobs jobs = {};
    jobs.job[0] = MapJob{p.bm[0], max_tiles_of(R, p.bm[0], nseg), tilemap_at(workspace, R)};
    jobs.job[1] = p.bm[1] == p.bm[0] ? jobs.job[0] : MapJob{p.bm[1], max_tiles_of(R, p.bm[1], nseg), tilemap_at(workspace, R, 1, jobs.job[0].max_tiles)};
    jobs.done = tilemap_at(workspace, R, 0, max_tiles_for(R) - 2).rel;
    jobs.job[0].m.done = jobs.done;
    jobs.job[1].m.done = jobs.done + kMaxSplitTiles;
    const int n_maps = p.bm[1] == p.bm[0] ? 1 : 2;
    if (nseg <= kSmallMapSegs) {
        const int blocks = std::min(64, (R / std::min(p.bm[0], p.bm[1]) + std::min(nseg, n_local) + 3) / 4);
        hipLaunchKernelGGL(tilemap_small_kernel<false>, dim3(blocks, n_maps), dim3(256), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
    } else {
        hipLaunchKernelGGL(tilemap_kernel, dim3(n_maps), dim3(kMapThreads), 0, st, seg_offset, seg_expert, nseg, R, n_local, gather, jobs);
    }
    MOE_LAUNCH_CHECK("tilemap_kernel");
    const TileMap &m = jobs.job[0].m, &m2 = jobs.job[1].m;
    float* const pieces = reinterpret_cast<float*>(reinterpret_cast<char*>(h) + align256((size_t)R * fp8_row_bytes(F)));
    int rc;
    if (p.mt) {
        const int tiles = (R + n_used * (p.bm[0] - 1)) / p.bm[0];   // at most
        if (act == MOE_ACT_SWIGLU) rc = launch_stream<EPI_SWIGLU>(p.mt, recv, m, tab, F, H, h, ldh, tiles, pieces, st);
        else if (act == MOE_ACT_GELU_MLP) rc = launch_stream<EPI_GELU>(p.mt, recv, m, tab, F, H, h, ldh, tiles, pieces, st);
        else rc = launch_stream<EPI_SILU>(p.mt, recv, m, tab, F, H, h, ldh, tiles, pieces, st);
        if (rc != MOE_OK) return rc;
        return launch_stream<EPI_PLAIN>(p.mt, h, m2, tab, H, F, out, H * 2, tiles, pieces, st);
    }
    if (act == MOE_ACT_SWIGLU) rc = launch_fp8<EPI_SWIGLU>(p.bm[0], recv, m, tab, 0, 1, F, H, h, ldh, R, nseg, n_used, false, nullptr, st);
    else if (act == MOE_ACT_GELU_MLP) rc = launch_fp8<EPI_GELU>(p.bm[0], recv, m, tab, 0, 0, F, H, h, ldh, R, nseg, n_used, false, nullptr, st);
    else rc = launch_fp8<EPI_SILU>(p.bm[0], recv, m, tab, 0, 0, F, H, h, ldh, R, nseg, n_used, false, nullptr, st);
    if (rc != MOE_OK) return rc;
    return launch_fp8<EPI_PLAIN>(p.bm[1], h, m2, tab, 2, 2, H, F, out, H * 2, R, nseg, n_used, p.deep, may_cut(F) ? pieces : nullptr, st);
}
