// What the expert FFNs share, whatever the type of their rows (ffn.hip, ffn_fp8.hip): the map of tiles of the received rows, the
// numbering of tiles over the chip, the cut of a last round along K, the walk of a block, the LDS layout of operand tiles.
#pragma once
#include "common.h"
#include <algorithm>
#include <cmath>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxSeg = 1024;

struct TileMap {
    int32_t* n_tiles;   // [1]
    int32_t* row0;      // [max_tiles] first row of the tile
    int32_t* nrows;     // [max_tiles] valid rows (1..BM)
    int32_t* expert;    // [max_tiles] local expert
    int32_t* gather;    // [max_tiles] 0: the tile is rows row0 .. row0 + nrows - 1; 1: row r is row0 + rel[tile][r]
    int32_t* rel;       // [max_tiles][kRelPitch] row offsets of the gathered tiles (written for those only)
    int32_t* done;      // [kMaxSplitTiles] pieces that have arrived, per tile cut along K (zeroed with the map)
};
constexpr int kMaxSplitTiles = 256;
constexpr int kRelPitch = 256;

struct ExpertTable {
    const void* w1[MOE_MAX_LOCAL];
    const void* w_up[MOE_MAX_LOCAL];
    const void* w_down[MOE_MAX_LOCAL];
};

__host__ __device__ inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int max_tiles_for(int R) { return R / 64 + 1 + kMaxSeg; }
inline size_t tilemap_bytes(int R) {
    return align256(256 + 4 * sizeof(int32_t) * (size_t)max_tiles_for(R)) + (size_t)max_tiles_for(R) * kRelPitch * sizeof(int32_t);
}

// the map whose tiles are the workspace's records from `first` on; `which` (0, 1) has a tile count of its own
TileMap tilemap_at(void* ws, int R, int which = 0, int first = 0) {
    TileMap m;
    char* p = reinterpret_cast<char*>(ws);
    const size_t n = (size_t)max_tiles_for(R);
    m.n_tiles = reinterpret_cast<int32_t*>(p) + which;
    m.row0 = reinterpret_cast<int32_t*>(p + 256);
    m.nrows = m.row0 + n;
    m.expert = m.nrows + n;
    m.gather = m.expert + n;
    m.rel = reinterpret_cast<int32_t*>(p + align256(256 + 4 * sizeof(int32_t) * n));
    m.row0 += first; m.nrows += first; m.expert += first; m.gather += first;
    m.rel += (size_t)first * kRelPitch;
    m.done = nullptr;
    return m;
}
inline int max_tiles_of(int R, int bm, int nseg) { return std::min((R + bm - 1) / bm + nseg, R); }   // a tile has a row at least

// Tile map.  The received rows come as segments (rows seg_offset[i] .. seg_offset[i+1] - 1 belong to local
// expert seg_expert[i]); with several sources and several local experts the segments of one expert are not
// adjacent, and a segment can be much shorter than a tile (160 rows per source and expert under the
// capacity rule of the Switch-shape workload), so cutting every segment into tiles of its own would leave
// most tiles half empty.  With `gather` the segments of an expert are chained in index order into one
// list of rows that is cut into full tiles: a tile whose rows are not consecutive in memory carries a
// table of row offsets (rel), which the GEMM uses for its A-operand addresses and its output rows.
// Without `gather` only adjacent segments of the same expert are merged (every tile is consecutive rows).
//
// Items are the clamped, non-empty segments in processing order; a group is a maximal chain of items of
// one expert whose rows increase (so offsets from the tile's first row are never negative); tiles never
// straddle groups.  Both constructions - this one, and the one of lists of up to 64 segments below - are written once
// for the device kernel and for the host self check.
struct SegWork {
    int lo[kMaxSeg], hi[kMaxSeg], exp[kMaxSeg];                            // items (rows lo .. hi - 1 of one expert)
    int v0[kMaxSeg];                                                       // position of the item's first row in its group
    int grp[kMaxSeg];                                                      // group of the item
    int gaps[kMaxSeg];                                                     // items up to and including this one that do not follow their predecessor in memory
    int g_first[kMaxSeg + 1], g_tile0[kMaxSeg + 1], g_rows[kMaxSeg];       // groups: first item, first tile, rows
    int raw_off[kMaxSeg + 1], raw_exp[kMaxSeg];                            // the caller's segment list (raw_off: scratch once the items exist)
    int cnt[MOE_MAX_LOCAL], pos[MOE_MAX_LOCAL];
    int n_items, n_groups, n_tiles;
};
constexpr int kMapThreads = 1024;       // one block: a thread per segment / item, 16 waves to hide the LDS latency of the searches

// The steps take (tid, nth) = this thread and the thread count where they run in parallel; a barrier
// separates them.  The host self check runs the same per-element functions with plain loops in place
// of the block-wide ballots and prefix sums of the device kernel.
// 1: an expert outside [0, n_local) (-1) or an empty row range (-2) marks a segment to be skipped
__host__ __device__ inline void tilemap_clean(SegWork& w, int nseg, int R, int n_local, int tid, int nth) {
    for (int i = tid; i < nseg; i += nth) {
        const int lo = w.raw_off[i] > 0 ? w.raw_off[i] : 0;
        const int hi = w.raw_off[i + 1] < R ? w.raw_off[i + 1] : R;
        const int e = w.raw_exp[i];
        if (!(e >= 0 && e < n_local)) w.raw_exp[i] = -1;
        else if (!(hi > lo)) w.raw_exp[i] = -2;             // no rows: neither an item nor the end of a run
    }
    for (int e = tid; e < n_local; e += nth) w.cnt[e] = 0;
}
// 2 (gather), host form: rank of every segment among the segments of its expert, and the count per expert
inline void tilemap_rank_host(SegWork& w, int nseg) {
    for (int i = 0; i < nseg; ++i) {
        const int e = w.raw_exp[i];
        if (e < 0) continue;
        w.v0[i] = w.cnt[e]++;                        // the rank is parked in v0 until step 4
    }
}
// 3 (gather), host form: where the items of every expert start
inline void tilemap_starts_host(SegWork& w, int n_local) {
    int p = 0;
    for (int e = 0; e < n_local; ++e) { w.pos[e] = p; p += w.cnt[e]; }
    w.n_items = p;
}
// 4 (gather): segment i becomes item pos[e] + rank
__host__ __device__ inline void tilemap_place(SegWork& w, int nseg, int R, int tid, int nth) {
    for (int i = tid; i < nseg; i += nth) {
        const int e = w.raw_exp[i];
        if (e < 0) continue;
        const int k = w.pos[e] + w.v0[i];
        w.lo[k] = w.raw_off[i] > 0 ? w.raw_off[i] : 0;
        w.hi[k] = w.raw_off[i + 1] < R ? w.raw_off[i + 1] : R;
        w.exp[k] = e;
    }
}
// 2-4 without gathering (one thread): adjacent segments of the same expert merged
__host__ __device__ inline void tilemap_merge(SegWork& w, int nseg, int R) {
    int ni = 0, i = 0;
    while (i < nseg) {
        const int e = w.raw_exp[i];
        if (e < 0) { ++i; continue; }
        int j = i + 1;
        while (j < nseg && (w.raw_exp[j] == e || w.raw_exp[j] == -2)) ++j;
        const int lo = w.raw_off[i] > 0 ? w.raw_off[i] : 0;
        const int hi = w.raw_off[j] < R ? w.raw_off[j] : R;
        if (hi > lo) { w.lo[ni] = lo; w.hi[ni] = hi; w.exp[ni] = e; ++ni; }
        i = j;
    }
    w.n_items = ni;
}
// 5: does item k open a group / does it leave a gap behind its predecessor
__host__ __device__ inline bool tilemap_opens(const SegWork& w, int k, bool gather) {
    return !(gather && k > 0 && w.exp[k] == w.exp[k - 1] && w.lo[k] >= w.hi[k - 1]);
}
__host__ __device__ inline bool tilemap_gap(const SegWork& w, int k, bool gather) {
    return !tilemap_opens(w, k, gather) && w.lo[k] != w.hi[k - 1];
}
// 5, host form: groups and their tiles
inline void tilemap_groups_host(SegWork& w, int BM, bool gather) {
    const int ni = w.n_items;
    int ng = 0, nt = 0, rows = 0, gaps = 0;
    for (int k = 0; k < ni; ++k) {
        if (tilemap_opens(w, k, gather)) {
            if (ng > 0) { w.g_rows[ng - 1] = rows; nt += (rows + BM - 1) / BM; }
            w.g_first[ng] = k; w.g_tile0[ng] = nt; rows = 0;
            ++ng;
        }
        gaps += tilemap_gap(w, k, gather) ? 1 : 0;
        w.gaps[k] = gaps;
        w.v0[k] = rows;
        w.grp[k] = ng - 1;
        rows += w.hi[k] - w.lo[k];
    }
    if (ng > 0) { w.g_rows[ng - 1] = rows; nt += (rows + BM - 1) / BM; }
    w.g_first[ng] = ni; w.g_tile0[ng] = nt;
    w.n_groups = ng;
    w.n_tiles = nt;
}

// item of group g that holds group row v: the largest item with v0 <= v
__host__ __device__ inline int tilemap_item_of(const SegWork& w, int g, int v) {
    int c = w.g_first[g], d = w.g_first[g + 1];
    while (d - c > 1) { const int mid = (c + d) >> 1; if (w.v0[mid] <= v) c = mid; else d = mid; }
    return c;
}
struct TileSpan { int v_lo, v_hi, first_item, row0, gather; };
// tile q of group g: its range of group rows, its first row in memory, whether its rows have gaps
__host__ __device__ inline TileSpan tilemap_span(const SegWork& w, int g, int q, int BM) {
    TileSpan s;
    s.v_lo = q * BM;
    s.v_hi = w.g_rows[g] < s.v_lo + BM ? w.g_rows[g] : s.v_lo + BM;
    s.first_item = tilemap_item_of(w, g, s.v_lo);
    const int last_item = tilemap_item_of(w, g, s.v_hi - 1);
    s.row0 = w.lo[s.first_item] + (s.v_lo - w.v0[s.first_item]);
    s.gather = (w.gaps[last_item] - w.gaps[s.first_item] > 0) ? 1 : 0;   // a gap in front of an item that starts inside the tile
    return s;
}
// 6: the record of tile t
__host__ __device__ inline void tilemap_tile(const SegWork& w, int t, int BM, const TileMap& m) {
    int a = 0, b = w.n_groups;                       // largest group with g_tile0 <= t
    while (b - a > 1) { const int mid = (a + b) >> 1; if (w.g_tile0[mid] <= t) a = mid; else b = mid; }
    const TileSpan s = tilemap_span(w, a, t - w.g_tile0[a], BM);
    m.row0[t] = s.row0;
    m.nrows[t] = s.v_hi - s.v_lo;
    m.expert[t] = w.exp[s.first_item];
    m.gather[t] = s.gather;
}
// 7: the offset tables, item by item.  Only the first and the last tile of an item can have gaps (the
// tiles in between lie inside the item); for each of the two, if it has gaps, the item's rows in it are a
// run of consecutive table entries with consecutive values: rel[dst + r] = val + r for r < cnt.
struct RelJob { int dst, cnt, val; };
__host__ __device__ inline void tilemap_rel_jobs(const SegWork& w, int k, int BM, int n_tiles, RelJob (&job)[2]) {
    job[0] = job[1] = RelJob{0, 0, 0};
    const int g = w.grp[k], len = w.hi[k] - w.lo[k];
    const int q_a = w.v0[k] / BM, q_b = (w.v0[k] + len - 1) / BM;
    for (int pass = 0; pass < 2; ++pass) {
        const int q = pass == 0 ? q_a : q_b;
        if (pass == 1 && q_b == q_a) break;
        const int tile = w.g_tile0[g] + q;
        if (tile >= n_tiles) continue;
        const TileSpan s = tilemap_span(w, g, q, BM);
        if (!s.gather) continue;
        const int v_a = w.v0[k] > s.v_lo ? w.v0[k] : s.v_lo;                 // the item's rows inside the tile
        const int v_b = w.v0[k] + len < s.v_hi ? w.v0[k] + len : s.v_hi;
        job[pass].dst = tile * kRelPitch + (v_a - s.v_lo);
        job[pass].cnt = v_b - v_a;
        job[pass].val = w.lo[k] + (v_a - w.v0[k]) - s.row0;
    }
}

// Barrier that orders LDS traffic only (lgkmcnt(0), then s_barrier): the steps of the map exchange data
// through LDS alone, and __syncthreads() would also wait for every global store to land.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0); vmcnt and expcnt untouched
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// exclusive prefix sums of three values per thread over the block; totals to every thread
struct Int3 { int a, b, c; };
__device__ __forceinline__ Int3 block_scan3(Int3 v, Int3* excl, int* wave_tot /* LDS [3][16] */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    Int3 incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int ua = __shfl_up(incl.a, o, 64), ub = __shfl_up(incl.b, o, 64), uc = __shfl_up(incl.c, o, 64);
        if (lane >= o) { incl.a += ua; incl.b += ub; incl.c += uc; }
    }
    lds_barrier();                                 // wave_tot may still be read from an earlier scan
    if (lane == 63) { wave_tot[wave] = incl.a; wave_tot[16 + wave] = incl.b; wave_tot[32 + wave] = incl.c; }
    lds_barrier();
    Int3 before = {0, 0, 0}, total = {0, 0, 0};
#pragma unroll
    for (int wv = 0; wv < nw; ++wv) {
        const int ta = wave_tot[wv], tb = wave_tot[16 + wv], tc = wave_tot[32 + wv];
        if (wv < wave) { before.a += ta; before.b += tb; before.c += tc; }
        total.a += ta; total.b += tb; total.c += tc;
    }
    excl->a = before.a + incl.a - v.a; excl->b = before.b + incl.b - v.b; excl->c = before.c + incl.c - v.c;
    return total;
}

// How the tiles of a GEMM are numbered over the XCDs (see tile_of_block)
constexpr int kFewestStripTiles = 192, kStripTiles = 3000;
struct Strips { int wide, more; };                           // `more` strips of wide + 1 columns, then strips of `wide`; wide = 0: bands
__host__ __device__ __forceinline__ Strips plan_strips(int tiles_m, int tiles_n) {
    const int total = tiles_m * tiles_n;
    if (total < kFewestStripTiles || total > kStripTiles || (tiles_m / 8 < 4 && tiles_n / 8 > tiles_m / 8)) return Strips{0, 0};
    const float patch = fminf(total * 0.125f, 32.f), width = fmaxf(sqrtf(patch), patch / tiles_m);
    const int strips = max(1, min(tiles_n, (int)(tiles_n / width + 0.5f)));
    return Strips{tiles_n / strips, tiles_n % strips};
}
// One block per map, a thread per segment.  The segment list is read into LDS in one round trip; the stable order
// by expert comes from wave ballots (segments of the same expert inside a wave) plus a scan over the 16
// waves; groups, positions inside the groups and the tiles of the groups come from two block-wide prefix
// sums; then one thread per tile writes the tile records and the items fill the offset tables.
struct MapJob { int bm, max_tiles; TileMap m; };
struct MapJobs { MapJob job[2]; int32_t* done; int32_t* strips; int tiles_n[2]; };   // the two GEMMs may take tiles of different heights; done: both GEMMs' counters or NULL; strips: two numbers per GEMM (see Strips); tiles_n: column tiles of the GEMMs that are numbered by tile_of_block, else 0
// lane g < 2 writes the strips of GEMM g if map `job` of `maps` is its map
__device__ __forceinline__ void write_strips(const MapJobs& jobs, int job, int maps, int n_tiles, int lane) {
    if (lane >= 2 || (maps == 2 && lane != job) || jobs.tiles_n[lane] == 0) return;
    const Strips p = plan_strips(n_tiles, jobs.tiles_n[lane]);
    int32_t* to = jobs.strips + 2 * lane;
    to[0] = p.wide;
    to[1] = p.more;
}
__device__ __forceinline__ void zero_done(int32_t* done, int tid, int nth) {
    if (done)
        for (int i = tid; i < 2 * kMaxSplitTiles; i += nth) done[i] = 0;
}

// Up to 64 segments (every local expert of every source of a layer of up to 64 experts): lane k of EVERY wave holds
// segment k and works out the whole list for itself with ballots, lane permutations and prefix sums - no LDS, no
// barrier - and the waves share out the tiles.  10 -> 4.7 us at 64 segments against the block-wide kernel below.
// The steps are written once over W, the 64 lanes: WaveLanes on the device, ArrayLanes in the host self check.
constexpr int kSmallMapSegs = 64;
struct SmallItem {
    int off0, off1, e;               // in: seg_offset[k], seg_offset[k + 1], seg_expert[k]; e: then the item's expert
    int lo, len, hi;                 // rows lo .. hi - 1
    int rank;                        // position of the segment among the items
    int incl, excl;                  // rows of the items up to and in front of this one
    int prev_e, prev_hi;
    int v0;                          // position of the item's first row in its group
    int end, rows, tiles, tincl;     // of the group that the item opens: one past its last item, rows, tiles; tiles up to it
    bool ok, opens;
};
struct WaveLanes {
    SmallItem mine;
    int lane;
    template <class F> __device__ __forceinline__ void each(F f) { f(mine, lane); }
    template <class F> __device__ __forceinline__ unsigned long long ballot(F f) const { return __ballot(f(mine, lane)); }
    __device__ __forceinline__ int at(int SmallItem::*v, int k) const { return __builtin_amdgcn_readlane(mine.*v, k); }
    __device__ __forceinline__ void move_to_rank(int SmallItem::*v) { mine.*v = __builtin_amdgcn_ds_permute(mine.rank * 4, mine.*v); }
    __device__ __forceinline__ int from(int SmallItem::*v, int l, const SmallItem&) const { return __shfl(mine.*v, l, 64); }
    // by data-parallel moves: a few clocks each, where a shuffle takes the way through the LDS crossbar
    __device__ __forceinline__ void from_below(int SmallItem::*v, int SmallItem::*to) { mine.*to = __builtin_amdgcn_update_dpp(mine.*v, mine.*v, 0x138, 0xf, 0xf, false); }   // wave_shr:1
    __device__ __forceinline__ void prefix(int SmallItem::*v, int SmallItem::*to) {   // inclusive
        int x = mine.*v;
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8: inside rows of 16 lanes
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15: the row below into rows 1 and 3
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31: the lower half into rows 2 and 3
        mine.*to = x;
    }
};
struct ArrayLanes {
    SmallItem it[64];
    template <class F> void each(F f) { for (int l = 0; l < 64; ++l) f(it[l], l); }
    template <class F> unsigned long long ballot(F f) const {
        unsigned long long m = 0;
        for (int l = 0; l < 64; ++l) m |= (unsigned long long)(f(it[l], l) ? 1 : 0) << l;
        return m;
    }
    int at(int SmallItem::*v, int k) const { return it[k].*v; }
    void move_to_rank(int SmallItem::*v) {
        int old[64];
        for (int l = 0; l < 64; ++l) old[l] = it[l].*v;
        for (int l = 0; l < 64; ++l) it[it[l].rank].*v = old[l];
    }
    int from(int SmallItem::*v, int l, const SmallItem&) const { return it[l].*v; }
    void from_below(int SmallItem::*v, int SmallItem::*to) { for (int l = 0; l < 64; ++l) it[l].*to = it[l > 0 ? l - 1 : 0].*v; }
    void prefix(int SmallItem::*v, int SmallItem::*to) {
        int x = 0;
        for (int l = 0; l < 64; ++l) it[l].*to = (x += it[l].*v);
    }
};
struct SmallMap {
    unsigned long long gaps;         // items that leave a gap behind their predecessor in the group
    int n_tiles;
};
template <class W>
__host__ __device__ __forceinline__ SmallMap small_map(W& w, int nseg, int R, int n_local, int gather, int BM, int max_tiles) {
    using U = unsigned long long;
    using S = SmallItem;
    w.each([&](S& s, int lane) {
        s.lo = s.off0 > 0 ? s.off0 : 0;
        const int hi = s.off1 < R ? s.off1 : R;
        s.len = hi > s.lo ? hi - s.lo : 0;                             // (of offsets that fall by 2^31 the difference would wrap)
        s.ok = lane < nseg && s.e >= 0 && s.e < n_local && s.len > 0;  // others are skipped
    });
    // items: the segments by (expert, index) - without gathering by index - first, the skipped ones behind them
    const U okm = w.ballot([](const S& s, int) { return s.ok; });
    const int ni = __builtin_popcountll(okm);
    U bit[6];                                                          // MOE_MAX_LOCAL = 64 experts: six bits
#pragma unroll
    for (int b = 0; b < 6; ++b) bit[b] = w.ballot([&](const S& s, int) { return s.ok && ((s.e >> b) & 1); });
    w.each([&](S& s, int lane) {
        const U below = (1ull << lane) - 1ull;
        U eq = okm, lt = 0;                                            // the items of this expert, of lower experts
#pragma unroll
        for (int b = 5; b >= 0; --b) {
            if ((s.e >> b) & 1) { lt |= eq & ~bit[b]; eq &= bit[b]; }
            else eq &= ~bit[b];
        }
        s.rank = gather ? __builtin_popcountll(lt) + __builtin_popcountll(eq & below) : __builtin_popcountll(okm & below);
        if (!s.ok) { s.rank = ni + __builtin_popcountll(~okm & below); s.len = 0; s.e = -1; }
    });
    w.move_to_rank(&S::lo);
    w.move_to_rank(&S::len);
    w.move_to_rank(&S::e);
    // groups: chains of items of one expert whose rows increase (without gathering: follow each other)
    w.prefix(&S::len, &S::incl);
    w.each([](S& s, int) { s.excl = s.incl - s.len; s.hi = s.lo + s.len; });
    const int total = w.at(&S::incl, 63);
    w.from_below(&S::e, &S::prev_e);
    w.from_below(&S::hi, &S::prev_hi);
    w.each([&](S& s, int lane) {
        s.opens = lane < ni && (lane == 0 || s.e != s.prev_e || (gather ? s.lo < s.prev_hi : s.lo != s.prev_hi));
    });
    SmallMap m;
    const U heads = w.ballot([](const S& s, int) { return s.opens; });
    m.gaps = w.ballot([&](const S& s, int lane) { return lane < ni && !s.opens && s.lo != s.prev_hi; });
    w.each([&](S& s, int lane) {
        const U upto = (2ull << lane) - 1ull, above = heads & ~upto;
        const int head = 63 - __builtin_clzll((heads & upto) | 1ull);  // bit 0 is set whenever there is an item
        s.v0 = s.excl - w.from(&S::excl, head, s);
        s.end = above ? __builtin_ctzll(above) : ni;
        const int excl_end = w.from(&S::excl, s.end < 63 ? s.end : 63, s);
        s.rows = (s.end < ni ? excl_end : total) - s.excl;
        s.tiles = s.opens ? (s.rows + BM - 1) / BM : 0;
    });
    w.prefix(&S::tiles, &S::tincl);
    // a well-formed list (non-decreasing offsets) stays below the bound; overlapping segments are cut off here
    const int nt = w.at(&S::tincl, 63);
    m.n_tiles = nt < max_tiles ? nt : max_tiles;
    return m;
}
// tile t: its record, the items that have rows in it and its range of group rows
struct SmallTile { int row0, nrows, expert, gather, v_lo; unsigned long long in; };
template <class W> __host__ __device__ __forceinline__ SmallTile small_tile(const W& w, const SmallMap& m, int t, int BM) {
    using S = SmallItem;
    SmallTile r;
    const int g = 63 - __builtin_clzll(w.ballot([&](const S& s, int) { return s.opens && s.tincl - s.tiles <= t; }));
    const int v_lo = (t - (w.at(&S::tincl, g) - w.at(&S::tiles, g))) * BM, rows = w.at(&S::rows, g), g_end = w.at(&S::end, g);
    const int v_hi = rows < v_lo + BM ? rows : v_lo + BM;
    r.in = w.ballot([&](const S& s, int lane) { return lane >= g && lane < g_end && s.v0 < v_hi && s.v0 + s.len > v_lo; });
    const int f = __builtin_ctzll(r.in);
    r.row0 = w.at(&S::lo, f) + v_lo - w.at(&S::v0, f);
    r.nrows = v_hi - v_lo;
    r.expert = w.at(&S::e, f);
    r.gather = (m.gaps & r.in & ~(1ull << f)) != 0 ? 1 : 0;            // a gap in front of an item that starts inside the tile
    r.v_lo = v_lo;
    return r;
}
// the table entries of item k of a gathered tile: rel[v] = val + v for lo <= v < hi
struct SmallRun { int lo, hi, val; };
template <class W> __host__ __device__ __forceinline__ SmallRun small_run(const W& w, const SmallTile& r, int k) {
    using S = SmallItem;
    const int v0 = w.at(&S::v0, k) - r.v_lo, hi = v0 + w.at(&S::len, k);
    return SmallRun{v0 > 0 ? v0 : 0, hi < r.nrows ? hi : r.nrows, w.at(&S::lo, k) - v0 - r.row0};
}

// STRIPS: a GEMM may be numbered in strips.  Without, the kernel is 0.5 us shorter, which shows in shares of 17 to 40 us.
template <bool STRIPS>
__global__ __launch_bounds__(256) void tilemap_small_kernel(const int32_t* __restrict__ seg_offset,
                                                            const int32_t* __restrict__ seg_expert, int nseg, int R,
                                                            int n_local, int gather, MapJobs jobs) {
    const MapJob& job = jobs.job[blockIdx.y];
    const TileMap m = job.m;
    const int wave_id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    WaveLanes w;
    w.lane = threadIdx.x & 63;
    const int i = min(w.lane, nseg - 1);
    w.mine.off0 = seg_offset[i];
    w.mine.off1 = seg_offset[i + 1];
    w.mine.e = seg_expert[i];
    if (blockIdx.x == 0 && blockIdx.y == 0) zero_done(jobs.done, threadIdx.x, 256);
    const SmallMap sm = small_map(w, nseg, R, n_local, gather, job.bm, job.max_tiles);
    if (blockIdx.x == 0 && threadIdx.x == 0) *m.n_tiles = sm.n_tiles;
    if (STRIPS && wave_id == (int)gridDim.x * 4 - 1) write_strips(jobs, blockIdx.y, gridDim.y, sm.n_tiles, w.lane);   // often without a tile
    for (int t = wave_id; t < sm.n_tiles; t += gridDim.x * 4) {
        const SmallTile r = small_tile(w, sm, t, job.bm);
        if (w.lane == 0) {
            m.row0[t] = r.row0;
            m.nrows[t] = r.nrows;
            m.expert[t] = r.expert;
            m.gather[t] = r.gather;
        }
        if (!r.gather) continue;
        for (unsigned long long in = r.in; in; in &= in - 1) {
            const SmallRun run = small_run(w, r, __builtin_ctzll(in));
            for (int v = run.lo + w.lane; v < run.hi; v += 64) m.rel[(size_t)t * kRelPitch + v] = run.val + v;
        }
    }
}

// The segment list itself, for shares that take gemm_f32_kernel twice: its blocks take one tile each and every wave works it
// out from the list, instead of a map by a launch of its own.  A small fp32 share (256 tokens, 517 rows of 64 -> 128 -> 64) is
// bound by its launches: 32.1 -> 27.9 us with six instead of seven.  In the narrow tiles of decode steps the same gained
// nothing: the list is cold in every kernel, and what the map's launches cost (2 x 4.7 us) the four GEMMs took longer.  Up to 64
// segments, and few tiles (see kListTiles).
struct SegList { const int32_t *offset, *expert; int nseg, R, n_local, gather, max_tiles; };
__device__ __forceinline__ SmallMap load_segments(const SegList& g, int bm, WaveLanes& w) {
    w.lane = threadIdx.x & 63;
    const int i = min(w.lane, g.nseg - 1);
    w.mine.off0 = g.offset[i];
    w.mine.off1 = g.offset[i + 1];
    w.mine.e = g.expert[i];
    return small_map(w, g.nseg, g.R, g.n_local, g.gather, bm, g.max_tiles);
}
// rows of a tile (in it: 0 .. nrows - 1) -> offsets from its first row
template <int N> __device__ __forceinline__ void segment_rows(const WaveLanes& w, const SmallTile& r, int (&row)[N]) {
    if (!r.gather) return;
    int off[N];
#pragma unroll
    for (int i = 0; i < N; ++i) off[i] = 0;
    for (unsigned long long in = r.in; in; in &= in - 1) {
        const SmallRun run = small_run(w, r, __builtin_ctzll(in));
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (row[i] >= run.lo && row[i] < run.hi) off[i] = run.val + row[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) row[i] = off[i];
}

__global__ __launch_bounds__(kMapThreads) void tilemap_kernel(const int32_t* __restrict__ seg_offset,
                                                              const int32_t* __restrict__ seg_expert, int nseg, int R,
                                                              int n_local, int gather, MapJobs jobs) {
    const int BM = jobs.job[blockIdx.x].bm, max_tiles = jobs.job[blockIdx.x].max_tiles;
    const TileMap m = jobs.job[blockIdx.x].m;
    if (blockIdx.x == 0) zero_done(jobs.done, threadIdx.x, blockDim.x);
    __shared__ SegWork w;
    __shared__ int wave_cnt[kMapThreads / 64][MOE_MAX_LOCAL];
    __shared__ int wave_tot[3 * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nth = blockDim.x, nw = nth >> 6;       // at least as many threads as segments (the launch sees to that)
    for (int i = tid; i <= nseg; i += nth) {
        w.raw_off[i] = seg_offset[i];
        if (i < nseg) w.raw_exp[i] = seg_expert[i];
    }
    for (int i = tid; i < (kMapThreads / 64) * MOE_MAX_LOCAL; i += nth) (&wave_cnt[0][0])[i] = 0;
    lds_barrier();
    tilemap_clean(w, nseg, R, n_local, tid, nth);
    lds_barrier();
    if (gather) {
        // rank among the segments of the same expert: inside the wave from ballots over the bits of the expert id
        const int e = tid < nseg ? w.raw_exp[tid] : -1;
        unsigned long long peers = __ballot(e >= 0);
#pragma unroll
        for (int b = 0; b < 6; ++b) {                // MOE_MAX_LOCAL = 64 experts: six bits
            const unsigned long long mb = __ballot((e >> b) & 1);
            peers &= ((e >> b) & 1) ? mb : ~mb;
        }
        const int rank_in_wave = __popcll(peers & ((1ull << lane) - 1ull));
        if (e >= 0 && rank_in_wave == 0) wave_cnt[wave][e] = __popcll(peers);
        lds_barrier();
        if (tid < n_local) {                         // exclusive scan over the waves, total per expert
            int run = 0;
#pragma unroll
            for (int wv = 0; wv < nw; ++wv) {
                const int c = wave_cnt[wv][tid];
                wave_cnt[wv][tid] = run;
                run += c;
            }
            w.cnt[tid] = run;
        }
        lds_barrier();
        if (e >= 0) w.v0[tid] = wave_cnt[wave][e] + rank_in_wave;
        if (wave == 0) {                             // where the items of every expert start
            const int c = lane < n_local ? w.cnt[lane] : 0;
            int incl = c;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(incl, o, 64);
                if (lane >= o) incl += up;
            }
            if (lane < n_local) w.pos[lane] = incl - c;
            if (lane == 63) w.n_items = incl;
        }
        lds_barrier();
        tilemap_place(w, nseg, R, tid, nth);
    } else if (tid == 0) {
        tilemap_merge(w, nseg, R);
    }
    lds_barrier();
    // groups: item tid opens one or not; prefix sums give the group of every item, the rows in front of it
    // and the gaps up to it
    const int ni = w.n_items;
    const bool live = tid < ni;
    const bool opens = live && tilemap_opens(w, tid, gather != 0);
    const bool gap = live && tilemap_gap(w, tid, gather != 0);
    const int len = live ? w.hi[tid] - w.lo[tid] : 0;
    Int3 ex;
    const Int3 tot = block_scan3(Int3{opens ? 1 : 0, len, gap ? 1 : 0}, &ex, wave_tot);
    const int ng = tot.a;
    int* rows_before = w.raw_off;                    // rows in front of each group (the raw list is no longer needed)
    if (live) {
        w.grp[tid] = ex.a + (opens ? 1 : 0) - 1;
        w.gaps[tid] = ex.c + (gap ? 1 : 0);
        if (opens) { w.g_first[ex.a] = tid; rows_before[ex.a] = ex.b; }
    }
    if (tid == 0) { w.g_first[ng] = ni; rows_before[ng] = tot.b; w.n_groups = ng; }
    lds_barrier();
    if (live) w.v0[tid] = ex.b - rows_before[w.grp[tid]];
    const int g_rows = tid < ng ? rows_before[tid + 1] - rows_before[tid] : 0;
    Int3 ex2;
    const Int3 tot2 = block_scan3(Int3{tid < ng ? (g_rows + BM - 1) / BM : 0, 0, 0}, &ex2, wave_tot);
    if (tid < ng) { w.g_rows[tid] = g_rows; w.g_tile0[tid] = ex2.a; }
    // a well-formed list (non-decreasing offsets) stays below the bound; overlapping segments are cut off here
    const int nt = tot2.a < max_tiles ? tot2.a : max_tiles;
    if (tid == 0) { w.g_tile0[ng] = tot2.a; w.n_tiles = nt; *m.n_tiles = nt; }
    write_strips(jobs, blockIdx.x, gridDim.x, nt, tid);
    lds_barrier();
    for (int t = tid; t < nt; t += nth) tilemap_tile(w, t, BM, m);
    if (!gather) return;
    // offset tables: every item works out its (at most two) runs of table entries; the runs are then parked
    // in LDS, over the item arrays that nobody needs any more, and written by whole waves, 64 entries a time
    RelJob job[2] = {{0, 0, 0}, {0, 0, 0}};
    if (live) tilemap_rel_jobs(w, tid, BM, nt, job);
    lds_barrier();
    static_assert(offsetof(SegWork, gaps) == 5 * kMaxSeg * sizeof(int), "the six item arrays must be contiguous");
    int* jd = &w.lo[0];                              // [2 * kMaxSeg] each
    int* jc = jd + 2 * kMaxSeg;
    int* jv = jc + 2 * kMaxSeg;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        jd[2 * tid + pass] = job[pass].dst;
        jc[2 * tid + pass] = job[pass].cnt;
        jv[2 * tid + pass] = job[pass].val;
    }
    lds_barrier();
    // the runs go round the waves (run j to wave j % nw) so that a short list still uses all of them; lane l of
    // wave w holds runs w + nw * l and w + nw * (64 + l), and the wave walks through them one at a time
    int d_reg[2], c_reg[2], v_reg[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = wave + nw * (64 * h + lane);
        d_reg[h] = jd[j];
        c_reg[h] = jc[j];
        v_reg[h] = jv[j];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        unsigned long long todo = __ballot(c_reg[h] > 0);
        while (todo) {
            const int src = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int dst = __builtin_amdgcn_readlane(d_reg[h], src), cnt = __builtin_amdgcn_readlane(c_reg[h], src);
            const int val = __builtin_amdgcn_readlane(v_reg[h], src);
            for (int r = lane; r < cnt; r += 64) m.rel[(size_t)dst + r] = val + r;
        }
    }
}

enum { EPI_PLAIN = 0, EPI_SILU = 1, EPI_GELU = 2, EPI_SWIGLU = 3 };

// Tile number `id` of `total` = tiles_m * tiles_n -> (tile_m, tile_n); a bijection for every shape.
// Blocks are handed to the 8 XCDs round-robin (XCD = id % 8), each XCD has its own L2, and all of them
// share the memory-side cache.  The map gives XCD x a band of tiles_m / 8 consecutive M-tiles and lets it
// walk ALL N-tiles for that band, in groups of 8 (then 4, 2, 1) M-tiles, M fastest: the blocks resident on an
// XCD form a patch of a few M-tiles by a few N-tiles (few distinct operand tiles in its L2), and the 8 XCDs
// sweep the N-tiles in step with each other, so a B tile fetched for one XCD is in the memory-side cache
// when the other seven ask for it and the A bands stay there for the whole sweep.  The tiles_m % 8
// M-tiles that do not fill a band come last, cut evenly over the XCDs.
__host__ __device__ __forceinline__ void tile_of_block_bands(int id, int tiles_m, int tiles_n, int* tm, int* tn) {
    const int x = id % 8, j = id / 8;                        // XCD and position in that XCD's sequence
    const int q = tiles_m / 8;                               // M-tiles per band
    const int band = q * tiles_n;                            // tiles of a band
    if (j < band) {
        // group heights: 8 as often as it fits, then the binary digits of the rest, so that a height always
        // divides the 32 blocks resident on an XCD (a 8 x 4, 4 x 8, ... patch with no straddling rows)
        int in_g = j, h = 8, first = 0, rest = q;
        while (true) {
            while (h > rest) h >>= 1;
            const int sz = h * tiles_n;
            if (in_g < sz) break;
            in_g -= sz; first += h; rest -= h;
        }
        *tm = q * x + first + in_g % h;
        *tn = in_g / h;
        return;
    }
    const int lm = tiles_m - 8 * q;                          // left-over M-tiles (lm >= 1 here)
    const int left = lm * tiles_n;
    const int v = x * (left / 8) + min(x, left % 8) + (j - band);
    *tm = 8 * q + v % lm;
    *tn = v / lm;
}
// With fewer than 32 M-tiles a band is at most three rows of tiles (patches of 1 x 32 or 2 x 16 tiles: 33 or
// 18 operand tiles for the 32 resident blocks instead of 12); when the N side has thicker bands the same
// numbering is used with the roles of M and N exchanged: XCD x owns a band of N-tiles and all XCDs sweep
// the M-tiles in step.  Measured at the 4096 -> 14336 -> 4096 shape: +7 % on both GEMMs at 2000 rows (bands
// of one row), +2.5 % at 6745 and 7900 rows (three rows), +1 % at 4147 and 5000 (two rows); with bands of
// four to seven rows the exchange gains or loses less than 1 %, so those keep the M bands.
//
// bf16 grids of kFewestStripTiles to kStripTiles tiles that N does not band (see plan_strips), of GEMMs with K of least_strip_k and more, are
// numbered in strips instead: XCD x gets
// the x-th eighth of the tiles in an order that cuts N into strips and goes through a strip row by row, so that the tiles resident
// on an XCD form a patch about as high as it is wide.  Bands -> strips on the kernels as they are, one FFN after the other: left-over
// M-tiles and low bands, 2741 rows of 1152 -> 2304 -> 1152 for four experts 48.1 -> 47.2 us, 12000 of 1408 -> 2048 -> 1408 SwiGLU for
// eight 208.3 -> 205.3, 2476 of 3584 -> 2560 -> 3584 111.2 -> 105.2; thick M bands, 16384 of 2048 -> 2816 -> 2048 SwiGLU 420.8 -> 409.8, 16318 of
// 1664 -> 2816 -> 1664 253.0 -> 249.8, 20571 of 4096 -> 14336 -> 4096 (second GEMM) the same.  33 shares 1.009 in the geometric mean, three of
// them 0.984 to 0.991.  (Where N has the thicker bands, each XCD reads weights of its own, which strips do not keep up: up to 7 %
// slower.  Outside the two limits nothing was gained.)  fp32: 11 shares of 128 x 128 tiles 0.997 to 1.005, so those keep the bands.
// Working the numbers below out in every block costs 0.4 us of a GEMM that takes 12 to 17, so the tile map holds them.
__host__ __device__ __forceinline__ void tile_of_block_strips(int id, int total, int tiles_m, Strips p, int* tm, int* tn) {
    const int x = id % 8, base = total / 8, extra = total % 8;
    const int v = x * base + min(x, extra) + id / 8;         // place in the order
    const int head = p.more * (p.wide + 1) * tiles_m;        // tiles of the wider strips
    const unsigned w = p.wide + (v < head ? 1 : 0), u = v < head ? v : v - head;
    const unsigned row = u / w, strip = row / (unsigned)tiles_m;
    *tm = (int)(row - strip * (unsigned)tiles_m);
    *tn = (v < head ? 0 : p.more * (p.wide + 1)) + (int)(strip * w + (u - row * w));
}
__host__ __device__ __forceinline__ void tile_of_block(int id, int total, int tiles_m, int tiles_n, Strips strips, int* tm, int* tn) {
    if (strips.wide > 0) tile_of_block_strips(id, total, tiles_m, strips, tm, tn);
    else if (tiles_m / 8 < 4 && tiles_n / 8 > tiles_m / 8) tile_of_block_bands(id, tiles_n, tiles_m, tn, tm);
    else tile_of_block_bands(id, tiles_m, tiles_n, tm, tn);
}

// Tail splitting.  The grid runs in rounds of `ncu` tiles (one block per CU); the tiles of a last,
// mostly empty round would leave most CUs idle for a whole tile time.  When that round has at most
// ncu / 2 tiles, each of them is cut along K into `parts` pieces that run as separate blocks
// (1/parts of a tile time) and write fp32 partial tiles, which are added in piece order before the
// epilogue - at 128 x 128 by the piece that arrives last (see last_piece), else by gemm_bf16_tail_kernel.
// Everything here depends only on the shapes, so results do not vary from run to run; another tile
// height or another cut adds the products of a row in another order, i.e. may round the last bit differently.
struct TailPlan {
    int n_full;        // tiles handled whole: ids [0, n_full)
    int n_tail;        // tiles cut in pieces: ids [n_full, n_full + n_tail)
    int parts;         // pieces per tail tile (1: no tail)
    int pairs_per;     // k-tile pairs per piece
};
__host__ __device__ __forceinline__ TailPlan plan_tail(int total, int ncu, int nk) {
    TailPlan p;
    p.n_full = total; p.n_tail = 0; p.parts = 1; p.pairs_per = nk / 2;
    const int rem = total % ncu;
    const int npairs = nk / 2;
    if (rem == 0) return p;
    // up to 8 pieces of at least 16 k-tiles (more only add partial tiles) but for the last one, which has four at least: of p <= 8
    // pieces of ceil(npairs / p) pairs, npairs >= 8 p, the last has (npairs - (p - 1)^2) / p > 1 of them.  2 or 3 pieces pay for the extra
    // pass only when a piece is still long (64 k-tiles)
    const int parts = min(min(ncu / rem, npairs / 8), 8);
    if (parts < 2 || (parts < 4 && npairs / parts < 32)) return p;
    p.pairs_per = (npairs + parts - 1) / parts;
    p.parts = (npairs + p.pairs_per - 1) / p.pairs_per;
    p.n_tail = rem;
    p.n_full = total - rem;
    return p;
}
// ... with a tail of at most `most_tail` tiles, which the launch has made room for; else none
__host__ __device__ __forceinline__ TailPlan plan_tail_upto(int most_tail, int total, int ncu, int nk) {
    const TailPlan p = plan_tail(total, ncu, nk);
    return p.n_tail <= most_tail ? p : TailPlan{total, 0, 1, nk / 2};
}

// Which items (tiles, then pieces) a block of the bf16 GEMM walks through: item, item + ncu, ... below end.  Place p of the
// ncu places works through items p, p + ncu, ... in runs of `walk`, a block for each.  The places' runs end one after the
// other, not all at once: whenever a run ends its CU is free for what other streams have queued.  Blocks start in the
// order of their numbers, and so do the runs of a generation end.  No cut when there are no more than `walk` rounds.
struct WalkRun { int item, end; };
__host__ __device__ __forceinline__ WalkRun walk_run(int block, int ncu, int walk, int n_items) {
    const int gen = block / ncu, place = block % ncu;
    const int ahead = n_items <= walk * ncu ? 0 : (ncu - 1 - place) * walk / ncu;   // rounds that this place's runs end early
    const int r0 = gen * walk - ahead, r1 = r0 + walk;
    const int first = (r0 > 0 ? r0 : 0) * ncu + place, end = r1 * ncu;
    return WalkRun{first, end < n_items ? end : n_items};
}

// An operand tile is stored as blocks of 16 rows; a block is 1 KB = 64 slots of
// 16 bytes and is filled by ONE wave-wide direct-to-LDS load (lane l fills slot l).
// Inside a block the rows are kept row-major (4 slots per row, so 4 neighbouring
// lanes fetch 64 contiguous bytes of one row from memory), with the 16-byte chunk
// index XOR-ed by -row/4:
//     slot(r, c) = 4*r + (c ^ (-(r >> 2) & 3)),   r = 0..15, c = 0..3.
// The LDS has 64 banks and serves a ds_read_b128 sixteen lanes at a time: lanes 0-3, 12-15 and 20-27 of the
// lower half, its others, and the same of the upper half.  Those of an MFMA operand read - one chunk of 16 rows, or chunk l / 16
// of row l % 16 - fall on 16 different values of slot % 16, i.e. on all 64 banks once.  (With r >> 2 in place of its
// negative the second kind of read takes twice as long: 256 x 256 tiles 5 % slower.)
__device__ __forceinline__ int slot_of(int r, int c) { return (r << 2) + (c ^ (-(r >> 2) & 3)); }
// inverse for the loading lane: which (row, chunk) of the block lane l must fetch
__device__ __forceinline__ void rc_of_slot(int l, int* r, int* c) {
    *r = l >> 2;
    *c = (l & 3) ^ (-(l >> 4) & 3);
}
// byte offset of (row, chunk) inside an operand tile
__device__ __forceinline__ int tile_off(int row, int c) { return ((row >> 4) << 10) + (slot_of(row & 15, c) << 4); }

__device__ __forceinline__ float fast_silu(float a) {
    return a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896f * a));
}
// tanh-form GELU: 0.5 a (1 + tanh(u)) = a * sigmoid(2u), u = sqrt(2/pi) (a + 0.044715 a^3); one exp2 and one rcp
// (the exponent -log2(e) * 2u = a * (k1 + k2 a^2) is formed with the constants folded: five plain operations around the two slow ones)
__device__ __forceinline__ float fast_gelu(float a) {
    const float k1 = -1.44269504088896f * 1.5957691216057308f, k2 = k1 * 0.044715f;
    const float arg = a * __builtin_fmaf(k2, a * a, k1);
    return a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(arg));
}
template <int EPI> __device__ __forceinline__ float activation_fast(float a, float b) {
    if (EPI == EPI_SILU) return fast_silu(a);
    if (EPI == EPI_GELU) return fast_gelu(a);
    if (EPI == EPI_SWIGLU) return fast_silu(a) * b;
    return a;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2 v = {lo, hi};
    const bf16x2 b = __builtin_convertvector(v, bf16x2);      // round to nearest even in hardware
    return *reinterpret_cast<const uint32_t*>(&b);
}

constexpr int kMaxCU = 256;                    // tail pieces per launch, at most: sizes the partial-tile workspace

// number of CUs of the current device (a round of the grid), at most kMaxCU
int round_size() {
    static int ncu = 0;
    if (ncu == 0) {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            n = kMaxCU;
        ncu = n < kMaxCU ? n : kMaxCU;
    }
    return ncu;
}

// blocks for up to max_items tiles and pieces, of which only the device knows the number
int walk_blocks(int max_items, int walk, int ncu) {
    const int rounds = (max_items + ncu - 1) / ncu;
    return (rounds <= walk ? 1 : (rounds + 2 * walk - 2) / walk) * ncu;
}

// The pieces of a tile that is cut along K.  Every piece writes its fp32 accumulators; at 128 x 128 (and in the
// weight-streaming kernels) the block that arrives last (a counter per tile, nobody waits) adds all pieces in piece
// order - its own is read back like the others, so the result does not depend on who was last - and finishes the
// tile.  A kernel of its own for the sums costs 4.5 us where there is nothing to add and 5-16 us where there is, each
// time behind a launch gap; the last block reads up to half a megabyte (32 pieces of a weight-streaming tile: 1 MB) in
// about as long, without the gap.  The larger tiles have 0.8 to 2 MB of pieces, which take one block 20 us and more (93
// against 108 us for the second GEMM at 4096 -> 14336 -> 4096 and 701 rows): those are added by gemm_bf16_tail_kernel,
// spread over the chip.
// The writers may sit on other XCDs, whose L2s do not see each other: pieces are stored and read with accesses of
// agent scope (sc1: written through, read past the L2), the counter is an agent-scope atomic, and a wave's stores have
// completed (vmcnt(0)) before its block counts.  The same with plain accesses between __threadfence()s was far
// slower: every fence writes back the whole L2 (54 against 17 us at 110 tiles of four pieces).
constexpr int kAgentScope = 16;                              // cache policy bits of a buffer access: sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t pieces_rsrc(const float* partial, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(partial), 0, bytes, 0x00027000);
}
__device__ __forceinline__ void store_piece(__amdgpu_buffer_rsrc_t r, int quad, const f32x4& v) {   // 16 bytes at quad * 16
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, quad * 16, 0, kAgentScope);
}
__device__ __forceinline__ f32x4 load_piece(__amdgpu_buffer_rsrc_t r, int quad) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, quad * 16, 0, kAgentScope));
}
__device__ __forceinline__ bool last_piece(int32_t* done, int parts, int* lds_flag) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);                        // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    if (threadIdx.x == 0) *lds_flag = __hip_atomic_fetch_add(done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    asm volatile("" ::: "memory");
    return *lds_flag != 0;
}

}  // namespace
