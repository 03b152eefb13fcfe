// What the expert FFNs on 8-bit rows and weights share (ffn_fp8.hip, ffn_int8.hip): tile shapes, the cut of a last round along K, streaming of the weights for few rows,
// and the choice among them.
#pragma once
#include "ffn_tiles.h"
#include "fp8.h"
#include <cmath>

namespace {

// Block tile of 64 MI rows x 64 NJ weight rows; the 4 waves are 2 x 2, a wave holds MI x NJ tiles of 32 x 32.  A stage is 64 bytes
// of K of every row, 2 P + 1 of them a ring: 160 KB at 4 x 4 and P = 2.
constexpr int kKt = 64;
// P: pairs of k-tiles that the ring has room for.  With P > 2 the loads do not run that far ahead today: where a trip ends, the registers of the scales' loads are taken
// over, and the compiler waits there for all loads but that trip's.
template <int MI, int NJ, int P> struct Geom8 {
    static constexpr int STAGES = 2 * P + 1;
    static constexpr int BM = 64 * MI, BN = 64 * NJ;
    static constexpr int A_BYTES = BM * kKt;
    static constexpr int STAGE = A_BYTES + BN * kKt;
    static constexpr int LDS = STAGES * STAGE;
    static constexpr int PER_CU = LDS <= 80 * 1024 ? 2 : 1;                 // blocks that share a CU
};
template <int EPI, int NJ> struct Out8 {
    static constexpr int NOUT = (EPI == EPI_SWIGLU) ? 32 * NJ : 64 * NJ;   // output columns per block
    static constexpr int NW = NOUT / 2;                                    // per wave
};

__device__ __forceinline__ float from_agpr(float a) {
    float v;
    asm("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
    return v;
}

// The tiles of a last round that leaves CUs idle are cut along K into `parts` pieces of `per` blocks of 128 (a multiple of 4: words of scales), which run
// beside each other, leave their sums in fp32 and are added in their order by a kernel behind (gemm_fp8_sum_kernel).  Only the second GEMM, whose sums need no
// activation.  Worth what it saves, 1.45 us a block, if that is more than the launch, and writing and reading the pieces (256 KB each): 12 us and 0.105 us a piece.
// 4096 -> 14336 -> 4096: 20571 rows, 16 tiles behind five full rounds, 988 -> 903 us and 6 for the sums; 2000 rows, 128 tiles, 152 -> 98 and 17.
struct Cut8 { int n_full, n_tail, parts, per; };
constexpr int kCutPieces = 256, kCutParts = 8;               // pieces per launch and per tile, at most
__host__ __device__ __forceinline__ Cut8 plan_cut(int total, int ncu, int blocks) {
    const int rem = total % ncu;
    if (rem > 0 && ncu <= kCutPieces) {
        const int parts = min(min(ncu / rem, blocks / 4), kCutParts);
        if (parts >= 2) {
            const int per = ((blocks + parts - 1) / parts + 3) & ~3, n = (blocks + per - 1) / per;
            if (n >= 2 && 1.45f * (blocks - per) > 12.f + 0.105f * (rem * n)) return Cut8{total - rem, rem, n, per};
        }
    }
    return Cut8{total, 0, 1, blocks};
}
// ... with at most `most` tiles cut, for which the launch has made room; else none
__host__ __device__ __forceinline__ Cut8 plan_cut_upto(int most, int total, int ncu, int blocks) {
    const Cut8 c = plan_cut(total, ncu, blocks);
    return c.n_tail <= most ? c : Cut8{total, 0, 1, blocks};
}

struct Item8 {
    int tail, piece;         // a piece of a cut tile: the tile's number among the cut ones, the piece; else piece = -1
    int blocks;              // of 128 of K
    int row0, nrows, n0;
    int expert;
    const int32_t* rel;      // row offsets of a gathered tile, else NULL
};

// Where the rows of a tile that a lane stores are: byte offset from the tile's first row, or past the end of the descriptor
__device__ __forceinline__ uint32_t row_offset(const Item8& t, int r, int ldc) {
    const int c = min(r, t.nrows - 1);
    const int q = t.rel ? t.rel[c] : c;
    return r < t.nrows ? (uint32_t)q * (uint32_t)ldc : 0xFFFFFF00u;
}

// Few rows per expert: a block takes some output columns, 16 a wave, and K or a piece of it
constexpr int kStreamPieces = 256;                           // pieces per launch, at most: sizes the workspace
// Chunk c (16 bytes) of row r of a stage lies at slot c ^ this: the 16 lanes that a read serves at a time (0-3, 12-15, 20-27 of a half wave, or its others; row
// lane % 16, chunk lane / 16 or 4 + lane / 16) fall on all 64 banks once.
__device__ __forceinline__ int stream_swizzle(int r) { return (r >> 1) & 7; }

// Pieces along K: as many as fill the chip's CUs with a block each, of at least four blocks of K
inline int stream_pieces(int tiles, int N, int K) { return std::max(1, std::min(kStreamPieces / (tiles * (N / 128)), K / FP8_BLOCK / 4)); }

// How a share is run: tiles of 16 mt rows that stream the weights (mt > 0), or tiles of bm[g] rows in GEMM g.  Measured on e4m3 rows, and used for integers as it is, whose kernels differ
// (no scales in the loop, rows of h by a kernel of their own, 64 columns a block; below).  The number of tiles is known on the device
// only, so the choice goes by an estimate, half a tile of padding per expert, and by what the kernels were measured to take (microseconds; 23 shares of 300 to
// 40000 rows, 1 to 8 experts, K of 512 to 14336; `blocks` of K of 128):
//   256 x 256 tiles, a CU each: a single round 6 + 1.3 blocks, else 8 + 1.45 blocks a round, 7 more for SiLU or GELU (of 256 columns; the whole epilogue of quantised
//   columns against that of bf16 ones); 11 blocks 20 to 25, 112 blocks 148 to 164;
//   how many rounds is exact for one expert, else 0.4 more than the tiles fill, two at least (1024 -> 4096 GELU, four experts, 10199 rows 128 instead of 134 us in tiles of 128, 20000 rows 242 and 224)
//   128 x 128, two on a CU: 3 + 0.72 blocks where a CU has one (+ 4 for an activation), else (4 + 1.35 blocks) tiles / 512; 11 blocks 10 and 18, 112 blocks 86 and 140.
//   A second GEMM of at most a tile per CU takes a ring of four pairs of k-tiles, a CU to itself: 701 rows of 4096 -> 14336 -> 4096 194 -> 180 us, 403 of 2048 -> 1408 -> 2048 33.3 -> 32.8
//   128 x 256 (SwiGLU, whose 128 gate and 128 up rows make the 128 columns that are quantised together): 3 + blocks, from the third round on
//   4 + 1.05 blocks; 16 blocks 19, 21 to 25 a round, 32 blocks 37
//   64 x 256 (SwiGLU, at most a tile per CU): 3 + 0.82 blocks; 403 rows of 2048 -> 1408 -> 2048, four experts 32.8 -> 30.0
//   and no less than the weights at 3.3 TB/s.
// Streaming (stream_us): 8 us and the weights at 4.6 TB/s, 10 % more per 16 rows that a tile has above 16, and 0.325, 0.4 or 0.55 of the weights' time for every further tile
// of 16, 32 or 64 rows of an expert; no less than the chain
// of three kernels, 12 us and 5 + mt for each round of blocks of each GEMM, or, in layers of H + F <= 2048 whose blocks run at once on every XCD, 12 + mt and 0.15 + 0.05 mt a block of K of
// either GEMM.  There tiles that do not stream take 2 us more than the estimate, and streaming is both the faster and, its products being exact, the more accurate: 256 -> 256 SiLU, 1 to 400 rows 14
// us in tiles of 16 and 17 in tiles of 128, 800 rows 15.4 (32) and 17.6; 512 -> 640 SwiGLU 16.5 and 19; 1024 -> 1024 GELU 18 and 21, 800 rows 20 (32) and 22.5.
// 4096 -> 14336 -> 4096 SwiGLU, one expert: 16 rows 46 us in tiles of 16, 64 rows 57 and 58 in tiles of 32 and 64 rows, 128 rows 85 and 65 (tiles of 128 rows 133), 256 rows 97 in tiles of 64, 93 in tiles of 128 and 256, 701 rows 250 and 173.
// 2048 -> 1408 -> 2048, four experts: 64 rows 22, 24, 28 in tiles of 16, 32, 64 rows (26 in tiles that do not stream), 400 rows 38, 27, 33 (28), 800 rows 68, 46, 35 (30).
// Up to three experts of larger layers take the tile that their rows fill, more experts and those small layers the one of the least estimate.  For large experts, where the former was measured, the two agree (4096 -> 14336, above); for
// small ones of one to three the estimate's tiles of 16 would be the faster: 2048 -> 1408 SwiGLU, 60 rows of one expert 25.0 as chosen and 21.2, 120 of two 28.1 and 23.0, 180 of three 28.0 and 24.3;
// 1024 -> 4096 GELU, 120 of two 29.6 and 21.9.  With four and more the choice is at most 3 us from the best of these.
// From 16 experts on, which the fit had not seen, it is up to 16 % from the best of the tiles (forced in turn): 64 of 2048 -> 1408 SwiGLU, 384 rows 138 us as chosen (16) and 119 in tiles of 128, 3000
// rows 163 (256 and 128) and 139 (128), 24576 rows 314 (256); 32 of 1024 -> 4096 GELU, 1000 rows 86 (32) and 79 (128), 20000 rows 273 (128 and 256) and 265 (256); 16 of 2048 -> 5632 SwiGLU, 600 rows 147 (256 and 128) and 125 (128), 5000 rows
// 258 (256) and 296 (128).
// Integers, every height forced in turn, weights beyond the caches: 4096 -> 14336 SwiGLU, one expert, 1 to 2000 rows (eight shares) and 5000 rows of four of 2048 -> 5632 within 2 % of the best; four
// of 2048 -> 1408 SwiGLU, 200 rows 27.1 us as chosen (16) and 24.7 in tiles of 32, 403 rows 29.4 (32) and 28.8 (64), 800 rows 39.2 (64 and 128, not streamed) and 32.9 (64, streamed); four of
// 1152 -> 2304 SiLU, 400 rows 27.8 (32) and 24.3 (64), 1000 and 2741 rows within 3 %; two of 1024 -> 4096 GELU, 120 rows 23.0 (64) and 19.9 (32); 64 of 2048 -> 1408, 384 rows 137 (16) and 122
// (64 and 128), 3000 rows 177 (256 and 128) and 150 (128); 16 of 2048 -> 5632, 600 rows 163 (256 and 128) and 139 (128).
struct Plan8 { int mt, bm[2]; bool deep; };
constexpr int kStreamRows = 1024;
double estimated_tiles(int R, int bm, int n_used) { return n_used <= 1 ? (R + bm - 1) / bm : std::max<double>(n_used, (double)R / bm + 0.5 * n_used); }
double tile_us(int bm, int R, int n_used, int N, int K, int act) {           // act: -1 for the second GEMM
    const double blocks = K / FP8_BLOCK, cus = 256.0;
    const int cols = act == MOE_ACT_SWIGLU ? 128 : bm == 256 ? 256 : 128;
    const double tiles = estimated_tiles(R, bm, n_used) * ((N + cols - 1) / cols);
    const bool simple = act == MOE_ACT_SILU_MLP || act == MOE_ACT_GELU_MLP;
    double us;
    if (bm == 256) {
        const Cut8 cut = act < 0 ? plan_cut((int)tiles, 256, (int)blocks) : Cut8{0, 0, 1, 0};
        if (cut.parts > 1) us = cut.n_full / 256 * (8 + 1.45 * blocks) + 8 + 1.45 * cut.per + 12 + 0.105 * cut.n_tail * cut.parts;
        else if (tiles <= cus) us = 6 + 1.3 * blocks + (simple ? 6 : act >= 0 ? 2 : 0);
        else us = (n_used > 1 ? std::max(2.0, tiles / cus + 0.4) : std::ceil(tiles / cus)) * (8 + 1.45 * blocks + (simple ? 7 : 0));
    } else if (bm == 64) {
        us = tiles <= cus ? 3 + 0.82 * blocks : 1e30;
    } else if (act == MOE_ACT_SWIGLU) {
        const double rounds = tiles / cus;
        us = rounds <= 1 ? 3 + blocks : rounds <= 2 ? 2 * (2 + blocks) : (rounds + 0.4) * (4 + 1.05 * blocks);
    } else {
        us = 3 + 0.72 * blocks + (simple ? 4 : 0);
        if (tiles > cus) us = std::max(us, tiles / (2 * cus) * (4 + 1.35 * blocks) + 1.5);
    }
    return std::max(us, (double)n_used * N * K * (act == MOE_ACT_SWIGLU ? 2 : 1) / 3.3e6);
}
bool is_brief(int H, int F) { return H + F <= 2048; }
double stream_us(int mt, int R, int n_used, int H, int F, int act) {
    const double weights = (double)n_used * H * F * (act == MOE_ACT_SWIGLU ? 3 : 2) / 4.6e6, tiles = estimated_tiles(R, 16 * mt, n_used);
    auto rounds = [&](int N) { const double x = tiles * (N / 128) / 256; return x <= 1 ? 1 : x + 0.4; };
    auto at_once = [&](int N) { return tiles * ((N / 128 + 7) / 8) <= 32; };
    if (is_brief(H, F) && at_once(F) && at_once(H)) return std::max(12 + mt + (0.15 + 0.05 * mt) * ((H + F) / FP8_BLOCK), 8 + weights * (1 + 0.1 * (mt - 1)));
    return std::max(12 + (5 + mt) * (rounds(F) + rounds(H)), 8 + weights * (1 + 0.1 * (mt - 1) + (0.25 + 0.075 * mt) * (tiles / n_used - 1)));
}
// Records of the workspace that the maps of tiles (one, if the heights are equal) and the two of counters leave
int free_records(int R, int nseg, int bm0, int bm1) { return max_tiles_for(R) - 2 - max_tiles_of(R, bm0, nseg) - (bm0 == bm1 ? 0 : max_tiles_of(R, bm1, nseg)); }
// most_k: the longest K that the kernels which stream the weights take
Plan8 plan_ffn8(int R, int n_used, int nseg, int H, int F, int act, bool gather, int most_k) {
    Plan8 p = {0, {256, 256}, false};
    double us = 2;
    for (int g = 0; g < 2; ++g) {
        const int N = g == 0 ? F : H, K = g == 0 ? H : F, a = g == 0 ? act : -1;
        const double large = tile_us(256, R, n_used, N, K, a), small = tile_us(128, R, n_used, N, K, a);
        if (small < large) p.bm[g] = 128;
        double least = std::min(small, large);
        if (a == MOE_ACT_SWIGLU) {
            const double smaller = tile_us(64, R, n_used, N, K, a);
            if (smaller < least) { p.bm[g] = 64; least = smaller; }
        }
        p.deep = a < 0 && p.bm[g] == 128 && estimated_tiles(R, 128, n_used) * (N / 128) <= 256;
        us += least;
    }
    if (gather && R <= kStreamRows && std::max(H, F) <= most_k) {
        const int per_expert = R / n_used;
        const bool brief = is_brief(H, F);
        if (brief) us += 2;                                  // what the tiles' estimate lacks there
        if (n_used < 4 && !brief) {
            const int mt = per_expert <= 12 ? 1 : per_expert <= 26 ? 2 : 4;
            if (stream_us(mt, R, n_used, H, F, act) < us) p.mt = mt;
        } else {
            for (int mt = 1; mt <= 4; mt *= 2) {
                const double t = stream_us(mt, R, n_used, H, F, act);
                if (t < us) { us = t; p.mt = mt; }
            }
        }
    }
    if (p.mt) p.bm[0] = p.bm[1] = 16 * p.mt;
    else if (p.bm[0] != p.bm[1] && free_records(R, nseg, p.bm[0], p.bm[1]) < 0) p.bm[0] = p.bm[1] = std::max(p.bm[0], p.bm[1]), p.deep = false;   // room for one map
    return p;
}

// whether the second GEMM may have tiles that are cut: a single one behind the full rounds is cut into the most pieces at the least cost
bool may_cut(int F) { return plan_cut(1, kCutPieces, F / FP8_BLOCK).n_tail > 0; }

}  // namespace
