// The norms behind and in front of a block, with the block's gate and residual scale between them, and the block's Aggregation in front where it is one
// of experts.
//
//   y = sum_j topk_w[t,j] ret[slot_to_row[t k + j]] (+ shared)        (or an array)
//   u = y / sqrt(mean y^2 + eps) gamma_post                            (or y)
//   r = round(residual + scale gate u);   v = r / sqrt(mean r^2 + eps) gamma_pre;   normed = round(v);   rows = v in 8 bits
//
// One pass: a row lives in the registers of W waves (8 neighbouring elements per lane and chunk of 512) from its loads, which all go out together, to its
// stores; sums and the largest element cross lanes by data-parallel moves and waves through LDS.  Bound by memory: every array once.
//
// Everything between the loads and the stores is 64 bits, as in the norm that feeds a share: r and the 8-bit rows are what the 64-bit numbers round to.
//
// bf16: 16384 rows of 2048 with integer rows 62 us (302 MB, 4.9 TB/s: the 64-bit arithmetic takes some 85 % of the cycles of the vector units, and is what is left; with a
// compare-and-select maximum, rint, shifts and divisions by the compiler's code it was 86); combined from six rows and a shared one, e4m3 rows 125 to 131 us (706 MB, 5.4 to 5.6 TB/s; with
// branches round the loads of arrays that may be missing 141); 16 rows of 4096 4.1 us, a launch.  Rows longer than 4096, whose arrays are not all loaded ahead: 8192 rows without and
// with integer rows, 4096 55 and 64 us (4.9 and 4.7 TB/s), 5120, five waves of two chunks, 104 and 131 (3.2, 2.9), 7168 115 and 146 (4.1, 3.6), 8192 113 and 145 (4.7, 4.2), 16384 230 and
// 291 (4.7, 4.2), 32768 400 and 499 (5.4, 4.9); 16 rows of 8192 4.8 and 5.7, of 32768 10.4 and 13.5.
#include "norm_rows.h"
#include "int8.h"
#include <type_traits>

namespace {

struct BlockArgs {
    const void *y, *residual, *gamma_post, *gate, *gamma_pre;
    const int32_t* slot_to_row;
    const float* topk_w;
    const void* shared;
    void *residual_out, *normed;
    uint8_t* rows;
    int64_t token0;                  // of the launch
    double inv_h;
    float scale, eps;
    int T, H, k, pitch, gate_tokens, norm_post;
};
enum { ROWS_NONE = -1 };

// A row of an array in a descriptor: elements behind its end, and of an array that is not there, are read as zeros and not written
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(const void* p, size_t byte, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(p)) + byte, 0, p ? bytes : 0u, 0x00027000);
}
// 8 neighbouring elements as they are stored
template <int DT> struct Raw8 {
    static constexpr int N = DT == MOE_BF16 ? 1 : 2;
    u32x4 q[N];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int i) {
#pragma unroll
        for (int n = 0; n < N; ++n) q[n] = __builtin_amdgcn_raw_buffer_load_b128(r, i * (DT == MOE_BF16 ? 2 : 4) + 16 * n, 0, 0);
    }
    // ones where there is no array
    __device__ __forceinline__ void load_or_ones(__amdgpu_buffer_rsrc_t r, int i, const void* p) {
        constexpr uint32_t ONE = DT == MOE_BF16 ? 0x3f803f80u : 0x3f800000u;
        load(r, i);
        if (!p)
#pragma unroll
            for (int n = 0; n < N; ++n) q[n] = u32x4{ONE, ONE, ONE, ONE};
    }
    __device__ __forceinline__ float at(int j) const {
        if (DT == MOE_BF16) return j & 1 ? __uint_as_float(q[0][j / 2] & 0xffff0000u) : bf16_bits_to_f32(q[0][j / 2] & 0xffffu);
        return __uint_as_float(q[j / 4 % N][j % 4]);
    }
};
constexpr int kStreaming = 2;        // cache policy bits of a buffer access: nt
template <int DT, int POLICY> __device__ __forceinline__ void store_row8(__amdgpu_buffer_rsrc_t r, int i, const float (&v)[8]) {
    if (DT == MOE_BF16) {
        const u32x4 q = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        __builtin_amdgcn_raw_buffer_store_b128(q, r, i * 2, 0, POLICY);
    } else {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const u32x4 q = {__float_as_uint(v[4 * n]), __float_as_uint(v[4 * n + 1]), __float_as_uint(v[4 * n + 2]), __float_as_uint(v[4 * n + 3])};
            __builtin_amdgcn_raw_buffer_store_b128(q, r, i * 4 + 16 * n, 0, POLICY);
        }
    }
}
// max(m, |v|) as one instruction (what the compiler makes of the functions turns each operand into itself first); the other one where one is NaN
__device__ __forceinline__ double max_abs(double m, double v) {
    double o;
    asm("v_max_f64 %0, %1, |%2|" : "=v"(o) : "v"(m), "v"(v));
    return o;
}
// What such an instruction writes may not be moved between lanes at once, and the compiler, which puts the waits in, does not look into it
__device__ __forceinline__ double settled(double m) {
    asm("s_nop 1" : "+v"(m));
    return m;
}
template <int CTRL> __device__ __forceinline__ double max_ror(double m) { return settled(max_abs(m, ror<CTRL>(m))); }
// towards() of eight: looked at together, as few have to be moved
__device__ __forceinline__ void towards8(float (&f)[8], const double (&d)[8]) {
    uint32_t least = 0x7fffu;
#pragma unroll
    for (int j = 0; j < 8; ++j) least = min(least, __float_as_uint(f[j]) & 0x7fffu);
    if (least == 0u)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = towards(f[j], d[j]);
}
__device__ __forceinline__ double wave_max(double m) {
    m = max_ror<0x121>(max_ror<0x122>(max_ror<0x124>(max_ror<0x128>(settled(m)))));
    return max_abs(max_abs(lane_of(m, 0), lane_of(m, 16)), max_abs(lane_of(m, 32), lane_of(m, 48)));
}
// Over the W <= 16 waves of a row, whose first is `first`: sum and maximum (of numbers without a sign).  A word of LDS per wave, other ones from call to call (one barrier
// each); the lanes read them again and again, 4, 8 or 16 side by side, which takes two, three or four steps to join.
template <bool MAX, int CTRL> __device__ __forceinline__ double join(double v) { return MAX ? max_ror<CTRL>(v) : v + ror<CTRL>(v); }
template <bool MAX> __device__ __forceinline__ double over_row(double v, double* part, int first, int W) {
    v = MAX ? wave_max(v) : wave_sum(v);
    if (W == 1) return v;
    const int lane = threadIdx.x & 63, period = W <= 4 ? 4 : W <= 8 ? 8 : 16, i = lane & (period - 1);
    if (lane == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = i < W ? part[first + i] : 0.0;
    if (period == 16) v = join<MAX, 0x128>(v);
    if (period >= 8) v = join<MAX, 0x124>(v);
    return lane_of(join<MAX, 0x121>(join<MAX, 0x122>(v)), 0);
}
// an infinite sum: finite elements become zeros, infinite ones NaN
__device__ __forceinline__ double norm_factor(double sum, double inv_h, double eps) {
    return sum < __builtin_huge_val() ? inverse_root(__builtin_fma(sum, inv_h, eps)) : sum > 0.0 ? 0.0 : sum;
}

// J: rows that are combined at a time, 0: y is an array.  FORM: of the 8-bit rows.  W waves per row, CH chunks per wave (chunk c of wave w: elements
// (c W + w) 512 ...); a block is 4 / W rows, one for W >= 3.  With a chunk per wave all loads go out before anything waits; with more, what an element meets
// later is loaded there, as registers are short.  v is formed where it is used, from r, so that only r lives on.
template <int CH> constexpr int kBlockThreads = CH == 1 ? 512 : 1024;
template <int DT, int CH, int J, int FORM>
__global__ __launch_bounds__(kBlockThreads<CH>) void block_norm_kernel(const BlockArgs a, int W) {
    constexpr bool EAGER = CH == 1;
    constexpr int B = DT == MOE_BF16 ? 2 : 4, L = EAGER ? 1 : 0;
    __shared__ double part[3][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_block = W < 3 ? 4 / W : 1, first = wave / W * W, w = wave - first, H = a.H;
    const int row = blockIdx.x * per_block + wave / W;
    const bool live = row < a.T;                             // the same for a wave; a dead one still meets the barriers
    const int t = __builtin_amdgcn_readfirstlane(live ? row : a.T - 1);
    const size_t base = (size_t)t * H * B;
    const uint32_t bytes = (uint32_t)H * B;
    const int gate_row = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a.token0 + t) / (uint32_t)a.gate_tokens));
    const __amdgpu_buffer_rsrc_t r_res = row_of(a.residual, base, bytes), r_post = row_of(a.gamma_post, 0, bytes), r_pre = row_of(a.gamma_pre, 0, bytes),
                                 r_gate = row_of(a.gate, (size_t)gate_row * H * B, bytes);
    auto element = [&](int c) { return (c * W + w) * 512 + lane * 8; };
    auto apart = [] { if (CH > 2) __builtin_amdgcn_sched_barrier(0); };   // between chunks: the loads of all of them at once do not fit the registers
    Raw8<DT> res0[L + 1], post0[L + 1], gate0[L + 1], pre0[L + 1];
    if (EAGER) {
        res0[0].load(r_res, element(0));
        post0[0].load_or_ones(r_post, element(0), a.gamma_post);
        gate0[0].load_or_ones(r_gate, element(0), a.gate);
        pre0[0].load_or_ones(r_pre, element(0), a.gamma_pre);
    }
    double y[CH][8];
    if constexpr (J == 0) {
        Raw8<DT> v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c].load(row_of(a.y, base, bytes), element(c));
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[c][j] = (double)v[c].at(j);
    } else {
        {
            Raw8<DT> v[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c].load(row_of(a.shared, base, bytes), element(c));
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) y[c][j] = (double)v[c].at(j);
        }
        for (int j0 = 0; j0 < a.k; j0 += J) {
            __amdgpu_buffer_rsrc_t from[J];
            float wt[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const size_t slot = (size_t)t * a.k + min(j0 + j, a.k - 1);
                const int r = __builtin_amdgcn_readfirstlane(j0 + j < a.k ? a.slot_to_row[slot] : -1);
                const float f = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(a.topk_w[slot])));
                from[j] = row_of(a.y, (size_t)max(r, 0) * bytes, r >= 0 ? bytes : 0u);          // of a dropped slot nothing is read
                wt[j] = r >= 0 ? f : 0.f;
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                Raw8<DT> v[J];
#pragma unroll
                for (int j = 0; j < J; ++j) v[j].load(from[j], element(c));
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[c][e] = __builtin_fma((double)wt[j], (double)v[j].at(e), y[c][e]);
                apart();
            }
        }
    }
    double factor = (double)a.scale;
    if (a.norm_post) {
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fma(y[c][j], y[c][j], sum);
        factor = norm_factor(over_row<false>(sum, part[0], first, W), a.inv_h, (double)a.eps) * factor;
    }
    float r[CH][8];
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = element(c);
        Raw8<DT> res = res0[0], post = post0[0], gate = gate0[0];
        if (!EAGER) {
            res.load(r_res, i);
            post.load_or_ones(r_post, i, a.gamma_post);
            gate.load_or_ones(r_gate, i, a.gate);
        }
        // behind the row's end everything is zero, but the factor may be infinite (fp32 rows may end behind a lane's fourth element)
        const double factor_lo = i < H ? factor : 0.0, factor_hi = DT == MOE_BF16 ? factor_lo : i + 4 < H ? factor : 0.0;
        auto add_up = [&](auto gated) {                        // bound by the number of operations: none for a gate that is not there
            double d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double u = y[c][j] * (j < 4 ? factor_lo : factor_hi) * (double)post.at(j);
                d[j] = decltype(gated)::value ? __builtin_fma(u, (double)gate.at(j), (double)res.at(j)) : u + (double)res.at(j);
                r[c][j] = (float)d[j];
            }
            if (DT == MOE_BF16) towards8(r[c], d);
        };
        if (a.gate) add_up(std::true_type{});
        else add_up(std::false_type{});
        if (DT == MOE_BF16)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t q = bf16_pair(r[c][j], r[c][j + 1]);
                r[c][j] = bf16_bits_to_f32(q & 0xffffu);
                r[c][j + 1] = __uint_as_float(q & 0xffff0000u);
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)r[c][j], (double)r[c][j], sum);
        apart();
    }
    if (live && a.residual_out)
#pragma unroll
        for (int c = 0; c < CH; ++c) store_row8<DT, kStreaming>(row_of(a.residual_out, base, bytes), element(c), r[c]);
    if (FORM == ROWS_NONE && !a.normed) return;
    double inv = norm_factor(over_row<false>(sum, part[1], first, W), a.inv_h, (double)a.eps);
    auto pre_of = [&](int c) {
        Raw8<DT> p = pre0[0];
        if (!EAGER) p.load_or_ones(r_pre, element(c), a.gamma_pre);
        return p;
    };
    auto v_of = [&](int c, const Raw8<DT>& p, int j) { return (double)r[c][j] * inv * (double)p.at(j); };
    double most = 0.0, odd = 0.0;                            // odd: NaN where there is an infinity or a NaN, which the maximum passes over
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int chunk = c * W + w, i = element(c), n = H - i;
        const Raw8<DT> p = pre_of(c);
        float f[8], g[8];
        double v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = v_of(c, p, j);
            f[j] = (float)v[j];
            if (DT == MOE_F32) g[j] = f[j];
            if (FORM == MOE_ROWS_INT8) {                     // (H is a multiple of 128 there)
                most = max_abs(most, v[j]);
                odd = __builtin_fma(v[j], 0.0, odd);
            }
        }
        if (DT == MOE_BF16 || FORM == MOE_ROWS_FP8) towards8(f, v);
        if (DT == MOE_BF16)
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = f[j];
        if (live && a.normed) store_row8<DT, 0>(row_of(a.normed, base, bytes), i, g);
        if (FORM == MOE_ROWS_FP8 && live && chunk * 512 < H) {   // H is a multiple of 128: 16 lanes have a whole block or none
            uint8_t* const out = a.rows + (size_t)t * a.pitch;
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, n > 0 ? abs_bits(f[j]) : 0u);
            m = max_of_16_lanes(m);
            const bool bad = fp8_block_is_nan(m);
            const uint32_t b = bad ? 127u : fp8_scale_byte(m);
            const float s = fp8_inverse_scale(b);
            if (n > 0) {
                uint2 q = make_uint2(fp8_pack4(f[0], f[1], f[2], f[3], s), fp8_pack4(f[4], f[5], f[6], f[7], s));
                if (bad) q = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
                *reinterpret_cast<uint2*>(out + i) = q;
            }
            // the four scale bytes of the chunk as one word; a block beyond H gives zero, as the padding is
            const uint32_t byte = n > 0 ? b : 0u;
            const uint32_t word = __builtin_amdgcn_readlane(byte, 0) | __builtin_amdgcn_readlane(byte, 16) << 8 | __builtin_amdgcn_readlane(byte, 32) << 16 |
                                  (uint32_t)__builtin_amdgcn_readlane(byte, 48) << 24;
            if (lane == 0) *reinterpret_cast<uint32_t*>(out + H + 4 * chunk) = word;
        }
        apart();
    }
    if (FORM == MOE_ROWS_FP8 && live)
        for (int i = (H + 511) / 512 + w * 64 + lane; i < (a.pitch - H) / 4; i += W * 64) *reinterpret_cast<uint32_t*>(a.rows + (size_t)t * a.pitch + H + 4 * i) = 0u;
    if (FORM == MOE_ROWS_INT8) {
        if (odd != 0.0) most = __builtin_huge_val();
        const Int8Scale s = int8_scale(over_row<true>(most, part[2], first, W));
        if (!live) return;
        uint8_t* const out = a.rows + (size_t)t * a.pitch;
        if (CH > 1) {                                        // v is formed again: two chunks and more of it, and r in 64 bits, do not fit the registers
            asm volatile("" : "+v"(inv));
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(r[c][j]));
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = element(c);
            const Raw8<DT> p = pre_of(c);
            if (i >= H) continue;
            uint2 q = make_uint2(int8_pack4<false>(v_of(c, p, 0), v_of(c, p, 1), v_of(c, p, 2), v_of(c, p, 3), s.inverse),
                                 int8_pack4<false>(v_of(c, p, 4), v_of(c, p, 5), v_of(c, p, 6), v_of(c, p, 7), s.inverse));
            if (s.inverse == 0.0) q = make_uint2(0u, 0u);
            *reinterpret_cast<uint2*>(out + i) = q;
            apart();
        }
        if (w == 0 && lane < (a.pitch - H) / 4) *reinterpret_cast<uint32_t*>(out + H + 4 * lane) = lane == 0 ? __float_as_uint(s.s) : 0u;
    }
}

template <int DT, int CH, int J, int FORM>
int launch_blocks(const BlockArgs& all, int W, hipStream_t st) {
    const int most = (int)(kLaunchThreads / (64 * W));
    const size_t row = (size_t)all.H * (DT == MOE_BF16 ? 2 : 4);
    for (int64_t t = 0; t < all.T; t += most) {
        BlockArgs a = all;
        a.token0 = t;
        a.T = (int)std::min<int64_t>(most, all.T - t);
        auto at = [&](const void* p) { return p ? reinterpret_cast<char*>(const_cast<void*>(p)) + t * row : nullptr; };
        if (J == 0) a.y = at(all.y);
        a.residual = at(all.residual);
        a.shared = at(all.shared);
        a.residual_out = at(all.residual_out);
        a.normed = at(all.normed);
        if (all.rows) a.rows = all.rows + (size_t)t * all.pitch;
        if (J > 0) { a.slot_to_row = all.slot_to_row + (size_t)t * all.k; a.topk_w = all.topk_w + (size_t)t * all.k; }
        hipLaunchKernelGGL((block_norm_kernel<DT, CH, J, FORM>), dim3(W < 3 ? (a.T * W + 3) / 4 : a.T), dim3(W < 3 ? 256 : 64 * W), 0, st, a, W);
        MOE_LAUNCH_CHECK("block_norm_kernel");
    }
    return MOE_OK;
}
template <int DT, int J, int FORM>
int launch_chunks(const BlockArgs& a, hipStream_t st) {
    const int chunks = (a.H + 511) / 512;                    // a chunk per wave where a block of 8 waves holds the row
    if (chunks <= 8) return launch_blocks<DT, 1, J, FORM>(a, chunks, st);
    if constexpr (J == 8) {
        return launch_chunks<DT, 4, FORM>(a, st);            // registers
    } else {
        if (chunks <= 32) return launch_blocks<DT, 2, J, FORM>(a, (chunks + 1) / 2, st);
        return launch_blocks<DT, 4, J == 0 ? 0 : 2, FORM>(a, 16, st);
    }
}
template <int DT, int J>
int launch_form(const BlockArgs& a, int form, hipStream_t st) {
    if (!a.rows) return launch_chunks<DT, J, ROWS_NONE>(a, st);
    return form == MOE_ROWS_INT8 ? launch_chunks<DT, J, MOE_ROWS_INT8>(a, st) : launch_chunks<DT, J, MOE_ROWS_FP8>(a, st);
}
template <int DT>
int launch_block(const BlockArgs& a, int form, hipStream_t st) {
    if (a.k == 0) return launch_form<DT, 0>(a, form, st);
    if (a.k <= 2) return launch_form<DT, 2>(a, form, st);
    return a.k <= 4 ? launch_form<DT, 4>(a, form, st) : launch_form<DT, 8>(a, form, st);
}

// The checks that both entry points share; the rest of `a` is the caller's
int check_block(const char* fn, BlockArgs& a, const moe_block_rule* rule, int32_t dtype, int32_t row_format) {
    if (!rule || (a.T != 0 && !a.residual_out && !a.normed && !a.rows)) return moe_set_error(MOE_EINVAL, "%s: NULL argument", fn);
    if (a.T < 0 || a.H <= 0) return moe_set_error(MOE_EINVAL, "%s: T >= 0 and H > 0 required", fn);
    if (!(rule->eps >= 0.f) || rule->eps > 3.4e38f || !(rule->scale >= -3.4e38f && rule->scale <= 3.4e38f))
        return moe_set_error(MOE_EINVAL, "%s: a finite scale and a finite eps >= 0 required", fn);
    if (rule->norm_post != 0 && rule->norm_post != 1) return moe_set_error(MOE_EINVAL, "%s: norm_post is 0 or 1", fn);
    if (!rule->norm_post && rule->gamma_post) return moe_set_error(MOE_EINVAL, "%s: gamma_post without norm_post", fn);
    if (dtype != MOE_F32 && dtype != MOE_BF16) return moe_set_error(MOE_EDTYPE, "%s: unknown dtype %d", fn, dtype);
    if (row_format != MOE_ROWS_FP8 && row_format != MOE_ROWS_INT8) return moe_set_error(MOE_EDTYPE, "%s: unknown row format %d", fn, row_format);
    if (a.H > kNormMaxH) return moe_set_error(MOE_ESHAPE, "%s: H <= %d required", fn, kNormMaxH);
    if (a.rows && a.H % FP8_BLOCK != 0) return moe_set_error(MOE_ESHAPE, "%s: packed rows need H to be a multiple of 128", fn);
    if (rule->gate && (rule->gate_rows < 1 || rule->gate_tokens < 1 || (int64_t)rule->gate_rows * rule->gate_tokens < a.T))
        return moe_set_error(MOE_ESHAPE, "%s: %d rows of the gate for %d tokens each do not cover %d tokens", fn, rule->gate_rows, rule->gate_tokens, a.T);
    if (((size_t)a.H * elem_size(dtype)) % 16 != 0) return moe_set_error(MOE_EALIGN, "%s: row size H*elem must be a multiple of 16 bytes", fn);
    for (const void* p : {a.y, a.residual, a.shared, (const void*)a.residual_out, (const void*)a.normed, (const void*)a.rows, rule->gamma_post, rule->gate, rule->gamma_pre})
        if (!aligned16(p)) return moe_set_error(MOE_EALIGN, "%s: arrays must be 16-byte aligned", fn);
    if (a.normed && a.normed == a.residual_out) return moe_set_error(MOE_EINVAL, "%s: normed and residual_out are the same array", fn);
    a.gamma_post = rule->gamma_post;
    a.gate = rule->gate;
    a.gamma_pre = rule->gamma_pre;
    a.gate_tokens = rule->gate ? rule->gate_tokens : 1;
    a.norm_post = rule->norm_post;
    a.scale = rule->scale;
    a.eps = rule->eps;
    a.inv_h = 1.0 / a.H;
    a.pitch = (int)(row_format == MOE_ROWS_INT8 ? int8_row_bytes(a.H) : fp8_row_bytes(a.H));
    return MOE_OK;
}

}  // namespace

extern "C" size_t moe_int8_row_bytes(int32_t H) { return H > 0 && H % FP8_BLOCK == 0 ? int8_row_bytes(H) : 0; }

extern "C" int moe_block_norm(const void* y, const void* residual, const moe_block_rule* rule, int32_t T, int32_t H, int32_t dtype, void* residual_out,
                              void* normed, void* rows, int32_t row_format, void* stream) {
    if (T != 0 && !y) return moe_set_error(MOE_EINVAL, "moe_block_norm: NULL argument");
    BlockArgs a = {};
    a.y = y; a.residual = residual; a.residual_out = residual_out; a.normed = normed; a.rows = reinterpret_cast<uint8_t*>(rows);
    a.T = T; a.H = H;
    if (const int rc = check_block("moe_block_norm", a, rule, dtype, row_format)) return rc;
    if (T == 0) return MOE_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return dtype == MOE_BF16 ? launch_block<MOE_BF16>(a, row_format, st) : launch_block<MOE_F32>(a, row_format, st);
}

extern "C" int moe_combine_norm(moe_ctx* ctx, const void* ret, const int32_t* slot_to_row, const float* topk_w, const void* shared_out, const void* residual,
                                const moe_block_rule* rule, void* residual_out, void* normed, void* rows, int32_t row_format, void* stream) {
    if (!ctx || !ret || !slot_to_row || !topk_w) return moe_set_error(MOE_EINVAL, "moe_combine_norm: NULL argument");
    BlockArgs a = {};
    a.y = ret; a.slot_to_row = slot_to_row; a.topk_w = topk_w; a.shared = shared_out;
    a.residual = residual; a.residual_out = residual_out; a.normed = normed; a.rows = reinterpret_cast<uint8_t*>(rows);
    a.T = ctx->s.T; a.H = ctx->s.H; a.k = ctx->s.k;
    if (const int rc = check_block("moe_combine_norm", a, rule, ctx->s.dtype, row_format)) return rc;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return ctx->s.dtype == MOE_BF16 ? launch_block<MOE_BF16>(a, row_format, st) : launch_block<MOE_F32>(a, row_format, st);
}
