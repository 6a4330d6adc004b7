// Product of E4M3 rows (a scale for each 128 channels) and an E4M3 weight (a scale for each block of 128 x 128):
//   out[t][i] = bias[i] + sum_b xs[t][b] ws[i / 128][b] sum_{j in b} x[t][j] w[i][j].
//
// A block's sum is made from zero and added to the running sum with its scales, in fp32.  Output channels are the rows of a
// tile and tokens its columns, so a lane holds one token, whose scale is one number, and 4 neighbouring channels.  The order
// of a block's 128 products is free: both operands take 16-byte pieces g and g + 4 of their row in lane group g.
//
// bf16 outputs: the matrix cores' 8-bit products, a block in one instruction (16x16x128).  It adds them in groups of 8 with
// the bits above 2^-13 of the group's largest product only (measured: a product 2^14 below another of its group is lost, one
// 2^13 below is kept whole; across groups sums are fp32).  On normal values the sums are off by 1.4e-5 of their size, a
// hundredth of what rounding to bf16 leaves; where a sum cancels, up to 7 * 2^-13 of its terms.  fp32 outputs: codes are
// turned to bf16, which is exact, and multiplied there at half the rate, with sums of 1e-8.
#include <algorithm>

#include "lq_e4m3.hpp"
#include "lq_internal.hpp"

namespace lq {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const char *x, *w;
    const float *xs, *ws, *bias;
    char *out;
    int64_t x_stride, w_stride, out_stride;     // bytes
    int64_t xs_stride;                          // floats
    int32_t tokens, n, k, blocks;               // blocks: of k
    int32_t out_bf16;
};

// 32 codes of a row, pieces g and g + 4 of a block, as operands
template <bool EXACT> struct Operand;
template <> struct Operand<false> {
    i32x8 v;
    __device__ __forceinline__ void set(const uint4 &a, const uint4 &b) {
        v = i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
    }
};
template <> struct Operand<true> {
    bf16x8 v[4];
    __device__ __forceinline__ void set(const uint4 &a, const uint4 &b) {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x2_t two = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j / 2], 1.0f, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j / 2], 1.0f, false);
                v[i][2 * j] = two[0];
                v[i][2 * j + 1] = two[1];
            }
    }
};
// a tile's sum over one block
__device__ __forceinline__ f32x4 block_product(const Operand<false> &w, const Operand<false> &x) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 block_product(const Operand<true> &w, const Operand<true> &x) {
    f32x4 p = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], x.v[i], p, 0, 0, 0);
    return p;
}

// 16 codes of a row, zeros past its end (loaded from within and then cleared: a choice between the row and a constant would be
// one between addresses, with the constant in scratch memory).
__device__ __forceinline__ uint4 piece(const char *row, int at, int k) {
    const uint4 v = *(const uint4 *)(row + min(at, k - 16));
    return at < k ? v : make_uint4(0, 0, 0, 0);
}

// ---- scales whose product fp32 does not hold -----------------------------------------
//
// x_scale * w_scale may be 0, denormal or infinite where with the block's sum it is a normal number.  The kernels multiply
// the scales first, in 32 bits, and keep the least product.  A wave whose least one is below the normal numbers, or whose sums
// are not finite (one channel of a token tells: an infinite product leaves none of them so), looks its scales over, and if there
// are such products it makes its tiles again, straight from memory, with these as mantissas and exponents apart.  The other
// products keep their bits: the same instructions in the same order.  (Making up for it in the loops cost the larger tiles
// their registers, masks of the lanes 1 to 18% of the time; the least product costs half an instruction a column.)
constexpr int ZERO = 0x060, DENORMAL = 0x090, NORMAL = 0x108, ANY = 0x3FF;
__device__ __forceinline__ bool is(float x, int classes) { return __builtin_amdgcn_classf(x, classes); }
__device__ __forceinline__ bool beyond(float xs, float ws) {
    return is(xs * ws, ANY - NORMAL) && is(xs, NORMAL | DENORMAL) && is(ws, NORMAL | DENORMAL);
}

// What that rare path needs, read anew where it begins: the kernel's arguments from memory and the lane from a count of lanes, so
// that nothing of them takes registers in the loops before (the path comes after all tiles for the same reason: behind each
// tile's stores some 30 more scalar registers were spilled).
struct Anew {
    ProductArgs a;
    int lane;
    __device__ __forceinline__ Anew() {
        auto p = (const ProductArgs *)__builtin_amdgcn_kernarg_segment_ptr();       // (the first argument)
        uint32_t all = ~0u;
        asm volatile("" : "+s"(p), "+s"(all));
        a = *p;
        lane = (int)__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
    }
};

// Whether a lane has such a product: lane l16 looks at token t + l16, the lane groups at every fourth block of k each.  Rows of
// zeros, as padded batches have them, lose nothing by a product that is too small.
__device__ __forceinline__ bool any_beyond(const Anew &n, int t, int wb) {
    const ProductArgs &a = n.a;
    t = min(t + (n.lane & 15), a.tokens - 1);
    const float *xs = a.xs + t * a.xs_stride, *ws = a.ws + min(wb, (a.n - 1) / BLOCK) * a.blocks;
    const char *x = a.x + t * a.x_stride;
    bool found = false;
#pragma unroll 4
    for (int b = n.lane >> 4; b < a.blocks; b += 4) {
        if (!beyond(xs[b], ws[b])) continue;
        uint32_t any = fabsf(xs[b] * ws[b]) > 1.0f;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            const uint4 v = piece(x, b * BLOCK + 16 * i, a.k);
            any |= (v.x | v.y | v.z | v.w) & 0x7F7F7F7Fu;
        }
        found |= any != 0;
    }
    return __builtin_amdgcn_ballot_w64(found) != 0;
}

// A tile of 16 x 16: lane l16 takes token t and row `row` of w, whose scales are those of block `wb` of rows.  Adds blocks first,
// first + step, ... to sum, `count` of them, counted round at `wrap`.
template <bool EXACT>
__device__ __forceinline__ f32x4 tile_apart(const Anew &n, int t, int row, int wb, int first, int step, int count, int wrap, f32x4 sum) {
    const ProductArgs &a = n.a;
    const int g = n.lane >> 4;
    t = min(t, a.tokens - 1);
    const char *x = a.x + t * a.x_stride, *w = a.w + min(row, a.n - 1) * a.w_stride;
    const float *xs = a.xs + t * a.xs_stride, *ws = a.ws + min(wb, (a.n - 1) / BLOCK) * a.blocks;
#pragma unroll 1
    for (int m = 0; m < count; ++m) {
        int b = first + m * step;
        if (b >= wrap) b -= wrap;
        const int at = b * BLOCK + 16 * g;
        Operand<EXACT> wo, xo;
        wo.set(piece(w, at, a.k), piece(w, at + 64, a.k));
        xo.set(piece(x, at, a.k), piece(x, at + 64, a.k));
        const f32x4 p = block_product(wo, xo);
        const float s = xs[b], u = ws[b], f = s * u;
        const bool apart = beyond(s, u);
        const float mantissa = __builtin_amdgcn_frexp_mantf(s) * __builtin_amdgcn_frexp_mantf(u);
        const int exponent = __builtin_amdgcn_frexp_expf(s) + __builtin_amdgcn_frexp_expf(u);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            sum[r] = apart ? sum[r] + __builtin_amdgcn_ldexpf(p[r] * mantissa, exponent) : fmaf(p[r], f, sum[r]);
    }
    return sum;
}

// 4 neighbouring channels of a token, from channel c on (rows start at multiples of 16 bytes).
__device__ __forceinline__ void store4(const ProductArgs &a, int t, int c, f32x4 v) {
    if (t >= a.tokens || c >= a.n) return;
    if (a.bias) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += a.bias[min(c + r, a.n - 1)];
    }
    char *at = a.out + t * a.out_stride + (int64_t)c * (a.out_bf16 ? 2 : 4);
    if (c + 4 <= a.n) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        if (a.out_bf16) store_tok<true, 4>(at, f);
        else store_tok<false, 4>(at, f);
        return;
    }
#pragma unroll
    for (int r = 0; r < 3; ++r) {
        if (c + r >= a.n) break;
        if (a.out_bf16) ((uint16_t *)at)[r] = (uint16_t)pk_bf16(v[r], v[r]);
        else ((float *)at)[r] = v[r];
    }
}

// ---- few tokens -------------------------------------------------------------------
//
// Bound: the weight's bytes.  A workgroup owns 16 CT channels of 16 TT tokens; its waves take the blocks of k in turn, AHEAD
// of them on their way, straight from memory into registers, and join their sums in LDS.  1 token x 4096 -> 12288 10.9 us with
// weights from HBM (4.6 TB/s), 9.8 with one weight call after call, which the last-level cache holds; 77 x 1552 -> 1000 fp32 4.4.
constexpr int WAVES = 8, AHEAD = 2;

template <bool EXACT, int TT, int CT>
__global__ __launch_bounds__(64 * WAVES) void product_few_kernel(ProductArgs a) {
    __shared__ f32x4 parts[WAVES][TT * CT][64];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c0 = blockIdx.x * 16 * CT, t0 = blockIdx.y * 16 * TT;
    const char *wrow[CT], *xrow[TT];
    const float *srow[TT];
#pragma unroll
    for (int i = 0; i < CT; ++i) wrow[i] = a.w + min(c0 + 16 * i + l16, a.n - 1) * a.w_stride;
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int t = min(t0 + 16 * j + l16, a.tokens - 1);
        xrow[j] = a.x + t * a.x_stride;
        srow[j] = a.xs + t * a.xs_stride;
    }
    f32x4 acc[CT][TT] = {};
    float low = 1.0f;               // the least product of scales
    struct Pieces {
        uint4 w[CT][2], x[TT][2];
        float ws[CT], s[TT];
    };
    // block b's pieces; past k (the end of a last block that is shorter) zeros
    auto load = [&](Pieces &o, int b, bool whole) {
        const int at = b * BLOCK + 16 * g;
        auto pieces = [&](const char *row, uint4 *p) {
            p[0] = whole ? *(const uint4 *)(row + at) : piece(row, at, a.k);
            p[1] = whole ? *(const uint4 *)(row + at + 64) : piece(row, at + 64, a.k);
        };
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            pieces(wrow[i], o.w[i]);
            o.ws[i] = a.ws[min(c0 + 16 * i, a.n - 1) / BLOCK * a.blocks + b];
        }
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            pieces(xrow[j], o.x[j]);
            o.s[j] = srow[j][b];
        }
    };
    auto add = [&](const Pieces &o) {
        // (x's operands are kept and the weight's made one at a time: the other way 2 x 4 tiles of fp32 spilled registers)
        Operand<EXACT> x[TT];
#pragma unroll
        for (int j = 0; j < TT; ++j) x[j].set(o.x[j][0], o.x[j][1]);
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            Operand<EXACT> w;
            w.set(o.w[i][0], o.w[i][1]);
#pragma unroll
            for (int j = 0; j < TT; ++j) {
                const f32x4 p = block_product(w, x[j]);
                const float f = o.s[j] * o.ws[i];
                low = fminf(low, fabsf(f));
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], f, acc[i][j][r]);
            }
        }
    };
    // This wave's blocks, from a start of the workgroup's own on: 1 token x 4096 -> 12288 13.0 -> 10.6 us, 4096 -> 4096 6.0 -> 4.9
    // when it was made.
    // (Why was not found: rows 128 bytes further apart change nothing, so it is not that rows meet in a few channels.)
    const int whole = a.k / BLOCK, start = whole ? (int)(blockIdx.x * 5u % (unsigned)whole) : 0;
    const int mine = wave < whole ? (whole - 1 - wave) / WAVES + 1 : 0;
    auto block = [&](int m) {
        const int b = m * WAVES + wave + start;
        return b < whole ? b : b - whole;
    };
    Pieces o[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (u < mine) load(o[u], block(u), true);
    for (int m = 0; m < mine; m += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (m + u < mine) add(o[u]);
            if (m + u + AHEAD < mine) load(o[u], block(m + u + AHEAD), true);
        }
    }
    if (whole < a.blocks && wave == whole % WAVES) {    // a last block that is shorter
        load(o[0], whole, false);
        add(o[0]);
    }
    bool again = is(low, ANY - NORMAL);
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) again |= !is(acc[i][j][0], NORMAL | DENORMAL | ZERO);
    again = __builtin_amdgcn_ballot_w64(again) != 0;
    if (again) {
        const Anew n;
        again = false;
#pragma unroll 1
        for (int tile = 0; tile < TT * CT; ++tile) again |= any_beyond(n, t0 + 16 * (tile % TT), (c0 + 16 * (tile / TT)) / BLOCK);
    }
    if (again) {
        const Anew n;
#pragma unroll 1
        for (int tile = 0; tile < TT * CT; ++tile) {
            const int c = c0 + 16 * (tile / TT), t = t0 + 16 * (tile % TT) + (n.lane & 15), row = c + (n.lane & 15);
            f32x4 v = tile_apart<EXACT>(n, t, row, c / BLOCK, wave + start, WAVES, mine, whole, f32x4{0, 0, 0, 0});
            if (whole < a.blocks && wave == whole % WAVES) v = tile_apart<EXACT>(n, t, row, c / BLOCK, whole, 0, 1, INT32_MAX, v);
            parts[wave][tile][n.lane] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int j = 0; j < TT; ++j) parts[wave][i * TT + j][lane] = acc[i][j];
    }
    __syncthreads();
    for (int e = tid; e < TT * CT * 64; e += 64 * WAVES) {
        const int tile = e >> 6, from = e & 63;
        f32x4 v = parts[0][tile][from];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += parts[i][tile][from];
        store4(a, t0 + 16 * (tile % TT) + (from & 15), c0 + 16 * (tile / TT) + 4 * (from >> 4), v);
    }
}

template <bool EXACT, int TT, int CT>
hipError_t launch_few(const ProductArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)((a.n - 1) / (16 * CT) + 1), (unsigned)((a.tokens - 1) / (16 * TT) + 1));
    hipLaunchKernelGGL((product_few_kernel<EXACT, TT, CT>), grid, dim3(64 * WAVES), 0, st, a);
    return hipGetLastError();
}

// The largest piece that leaves 160 workgroups: fewer of them re-read less, and 16 x 16 where none does.  Up to 4 tokens the
// rows of x cost nothing.  (4096 x 4096: 16 tokens 6.9 us by 16 x 16, 12.4 by 16 x 64; 64 tokens 12.0 by 32 x 32, 15.8 by
// 32 x 64.  4096 x 12288: 16 tokens 12.8 by 16 x 64, 15.7 by 16 x 16; 1 token 11.0 and 9.8.)
template <bool EXACT>
hipError_t launch_few_tokens(const ProductArgs &a, hipStream_t st) {
    const int64_t t = (a.tokens - 1) / 16 + 1, c = (a.n - 1) / 16 + 1;
    auto fits = [&](int tt, int ct) { return a.tokens > 4 && t >= tt && c >= ct && ((t + tt - 1) / tt) * ((c + ct - 1) / ct) >= 160; };
    if (fits(2, 4)) return launch_few<EXACT, 2, 4>(a, st);
    if (fits(2, 2)) return launch_few<EXACT, 2, 2>(a, st);
    if (fits(1, 4)) return launch_few<EXACT, 1, 4>(a, st);
    if (fits(1, 2)) return launch_few<EXACT, 1, 2>(a, st);
    return launch_few<EXACT, 1, 1>(a, st);
}

// ---- many tokens ------------------------------------------------------------------
//
// Bound: issue, of matrix and vector instructions, which hardly overlap (32 cycles for a tile's products over a block, 8 for
// its 4 sums a lane), and the waves' meeting once a block; bytes for 256 tokens and less.  A workgroup owns a tile of
// 16 WT TJ tokens x 16 WC TI channels, a wave TJ x TI tiles of 16 x 16, all sums in registers.  Blocks of k are copied straight
// into LDS, STAGES - 1 ahead; a row's 8 pieces are placed by an exclusive or with bits of the row, so that the 16 rows that a
// read takes at once lie in 16 different places of a 256-byte line of banks.  Channels are dealt to a wave's tiles so that a
// lane ends up with 16 bytes of neighbouring outputs of a token at a time, and 4 lanes with 64.
//
// 8192 x 4096 -> 12288 bf16 377-385 us (2.1 PFLOP/s; the matrix cores are busy 53% of the cycles).  A version before the last
// steps without the outputs' stores 376, without copies too 298-338, without the waves' meeting too 259.  Two waves a SIMD: one
// with twice the tile took 480.  256 x 4096 -> 12288 24 us; 1531 x 4096 -> 4096 fp32 54-55, where the
// codes' conversions take as long as the products.

// Copies into LDS as dma16's and dma_element's: 16 bytes per lane from a uniform base and a lane's offset, and one element.
// Nothing is copied where `left` is not positive: no lane is on then (all are where these are called).  By the mask and
// not by a branch, so that the products around them stay one run of instructions.
__device__ __forceinline__ void dma16_if(int left, uint64_t base, uint32_t offset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_cmp_gt_i32 %3, 0\n\ts_cselect_b64 exec, -1, 0\n\t"
                 "global_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" :: "v"(offset), "s"(base), "s"(lds_base), "s"(left) : "memory", "scc");
}
__device__ __forceinline__ void dma4_if(int left, uint64_t base, uint32_t offset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_cmp_gt_i32 %3, 0\n\ts_cselect_b64 exec, -1, 0\n\t"
                 "global_load_lds_dword %0, %1\n\ts_mov_b64 exec, -1" :: "v"(offset), "s"(base), "s"(lds_base), "s"(left) : "memory", "scc");
}
// Waits until at most `few` (which 1) or `many` (which 2) copies and stores are under way, or none (which 0).
template <int FEW, int MANY>
__device__ __forceinline__ void wait_copies(int which) {
    asm volatile("s_cmp_gt_i32 %2, 1\n\ts_cbranch_scc1 2f\n\ts_cmp_gt_i32 %2, 0\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(0)\n"
                 "1:\n\ts_waitcnt vmcnt(%0)\n2:\n\ts_waitcnt vmcnt(%1)" :: "n"(FEW), "n"(MANY), "s"(which) : "memory", "scc");
}

template <int WT, int WC, int TJ, int TI, int STAGES>
struct Tile {
    static constexpr int WAVES = WT * WC, TOKENS = 16 * WT * TJ, CHANNELS = 16 * WC * TI;
    static constexpr int X_COPIES = TOKENS / 8 / WAVES, W_COPIES = CHANNELS / 8 / WAVES;   // of 8 rows, per wave
    static constexpr int COPIES = X_COPIES + W_COPIES + 1;                                 // ... and one of scales
    // (two stages leave the last copies little time, so they go in the first columns)
    static constexpr int PARTS = STAGES == 2 ? (TJ + 1) / 2 : TJ - 1, PER_PART = (COPIES + PARTS - 1) / PARTS;
    static constexpr int STAGE = (TOKENS + CHANNELS) * BLOCK;
    static constexpr int SCALES = TOKENS + 64;      // of the tokens, then of the weight's blocks beside them
    static_assert(TOKENS % (8 * WAVES) == 0 && CHANNELS % (8 * WAVES) == 0 && TOKENS % 64 == 0, "whole copies");
    static_assert(TOKENS / 64 < WAVES, "a wave is left for the weight's scales");
    static_assert(TJ % 2 == 0 && TI % 2 == 0, "columns take turns in two registers, tiles of bf16 outputs go in pairs");
};

// Row m of a wave's tile i among its 16 TI rows of w, and the bits that place a row's pieces: those of m / 2, as for the rows
// of x.  (LDS serves a 16-byte read in groups of 16 lanes that take 8 rows of one lane group and the other 8 of the next; with
// the bits of m / 2 in another order a fifth of the LDS's active cycles were conflicts.)
template <bool EXACT>
__device__ __forceinline__ int tile_row(int i, int m) { return EXACT ? 16 * i + m : 32 * (i >> 1) + 8 * (m >> 2) + 4 * (i & 1) + (m & 3); }
template <bool EXACT>
__device__ __forceinline__ int row_place(int row) { return EXACT ? row >> 1 & 7 : (row >> 3 & 3) << 1 | (row >> 1 & 1); }

template <bool EXACT, int WT, int WC, int TJ, int TI, int STAGES>
__global__ __launch_bounds__(64 * WT * WC) void product_kernel(ProductArgs a, int tiles_t, int tiles_c) {
    using T = Tile<WT, WC, TJ, TI, STAGES>;
    __shared__ __attribute__((aligned(1024))) char codes[STAGES][T::STAGE];     // rows of x, then of w
    __shared__ float scales[STAGES][T::SCALES];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / WC, wc = wave % WC;
    const int whole = a.k / BLOCK, total = tiles_t * tiles_c;

    // Workgroups go round the 8 XCDs: each gets neighbouring tiles, a band of GROUP tiles of tokens side by side, whose rows its
    // L2 shares.  Bands start an eighth of the channels apart: where all XCDs walked the weight's rows alike, 8192 x 1024 ->
    // 12288 took 142 instead of 126 us, 4096 -> 12288 440 and 400.
    struct Place {
        int t0, c0;
    };
    auto place = [&](int turn) {
        constexpr int GROUP = 4;
        const int xcd = turn % 8, id = xcd * (total / 8) + min(xcd, total % 8) + turn / 8;
        const int band = id / (GROUP * tiles_c), first = band * GROUP, high = min(GROUP, tiles_t - first);
        const int in_band = id - band * GROUP * tiles_c;
        const int t = (first + in_band % high) * T::TOKENS, c = (in_band / high + band * (tiles_c / 8)) % tiles_c * T::CHANNELS;
        // (divisions are made in vector registers)
        return Place{__builtin_amdgcn_readfirstlane(t), __builtin_amdgcn_readfirstlane(c)};
    };

    // ---- copies: the blocks of this workgroup's tiles, one after the other ----
    const int row8 = lane >> 3, slot = lane & 7;
    auto piece_x = [&](int i) { return 16 * (slot ^ (8 * (wave * T::X_COPIES + i) + row8 >> 1 & 7)); };
    auto piece_w = [&](int i) { return 16 * (slot ^ row_place<EXACT>(8 * (wave * T::W_COPIES + i) + row8)); };
    uint32_t xo[T::X_COPIES], wo[T::W_COPIES];      // this lane's rows and pieces
    uint32_t so;
    uint64_t xbase, wbase, sbase;
    int kb = 0;                                     // the next block of k to send
    int to_copy = 0, copied = 0, place_of_copy = 0; // blocks of the tile not sent yet, blocks sent in all, their place in LDS
    int turn = blockIdx.x - gridDim.x;
    auto next_tile = [&]() {                        // the copies go on with the next tile, if there is one
        if (to_copy > 0 || turn + (int)gridDim.x >= total) return;
        turn += gridDim.x;
        const Place at = place(turn);
#pragma unroll
        for (int i = 0; i < T::X_COPIES; ++i)
            xo[i] = (uint32_t)(min(8 * (wave * T::X_COPIES + i) + row8, a.tokens - 1 - at.t0) * a.x_stride) + piece_x(i);
#pragma unroll
        for (int i = 0; i < T::W_COPIES; ++i)
            wo[i] = (uint32_t)(min(8 * (wave * T::W_COPIES + i) + row8, a.n - 1 - at.c0) * a.w_stride) + piece_w(i);
        xbase = (uint64_t)(a.x + at.t0 * a.x_stride);
        wbase = (uint64_t)(a.w + at.c0 * a.w_stride);
        if (wave < T::TOKENS / 64) {
            sbase = (uint64_t)(a.xs + at.t0 * a.xs_stride);
            so = (uint32_t)(min(64 * wave + lane, a.tokens - 1 - at.t0) * a.xs_stride * 4);
        } else {
            sbase = (uint64_t)a.ws;
            // (a copy costs the lines that it touches: with 64 blocks here instead of the tile's one or two, 256 x 4096 ->
            // 12288, weights that were in no cache, took 38.5 instead of 31.4 us)
            const int block = at.c0 / BLOCK + min(lane, (T::CHANNELS - 1) / BLOCK);
            so = (uint32_t)min(block, (a.n - 1) / BLOCK) * (uint32_t)a.blocks * 4u;
        }
        kb = 0;
        to_copy = a.blocks;
    };
    const uint32_t xl = lds_addr(codes) + wave * T::X_COPIES * 1024, wl = lds_addr(codes) + T::TOKENS * BLOCK + wave * T::W_COPIES * 1024;
    const uint32_t sl = lds_addr(scales) + 256 * min(wave, T::TOKENS / 64);
    // The next block on its way, in PARTS parts (nothing if there is none).  A part a column of products: sent all at once they
    // take the address units longer than a column lasts, and the waves wait to issue.
    auto copy_part = [&](int left, int part) {
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) {
            if (i / T::PER_PART != part) continue;
            if (i < T::X_COPIES)
                dma16_if(left, xbase + (uint64_t)kb * BLOCK, xo[i], xl + place_of_copy * T::STAGE + 1024 * i);
            else if (i < T::X_COPIES + T::W_COPIES)
                dma16_if(left, wbase + (uint64_t)kb * BLOCK, wo[i - T::X_COPIES], wl + place_of_copy * T::STAGE + 1024 * (i - T::X_COPIES));
            else
                dma4_if(left, sbase + (uint64_t)kb * 4, so, sl + place_of_copy * (T::SCALES * 4));
        }
    };
    // The last block, where k ends inside it, all at once: zeros past k, in places that nobody reads any more.  (Each row has
    // pieces before k, so every copy has lanes and is counted.)
    auto copy_short = [&]() {
        const int end = a.k - whole * BLOCK, st = place_of_copy;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const char *x = (const char *)xbase + whole * BLOCK, *w = (const char *)wbase + whole * BLOCK;
        char *xz = codes[st] + wave * T::X_COPIES * 1024 + 16 * lane, *wz = codes[st] + (T::TOKENS * BLOCK + wave * T::W_COPIES * 1024) + 16 * lane;
#pragma unroll
        for (int i = 0; i < T::X_COPIES; ++i) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(xl + st * T::STAGE + 1024 * i);
            if (piece_x(i) < end) dma16(x + xo[i], to);
            else *(uint4 *)(xz + 1024 * i) = zero;
        }
#pragma unroll
        for (int i = 0; i < T::W_COPIES; ++i) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(wl + st * T::STAGE + 1024 * i);
            if (piece_w(i) < end) dma16(w + wo[i], to);
            else *(uint4 *)(wz + 1024 * i) = zero;
        }
        dma4_if(1, sbase + (uint64_t)kb * 4, so, sl + st * (T::SCALES * 4));
    };
    auto copy_done = [&]() {
        ++kb;
        --to_copy;
        place_of_copy = place_of_copy + 1 == STAGES ? 0 : place_of_copy + 1;
    };
    // Before a block's parts: how many blocks are left, 0 if there is nothing to send in parts.
    auto copy_begin = [&]() {
        next_tile();
        if (to_copy <= 0) return 0;
        ++copied;
        if (kb < whole) return to_copy;
        copy_short();
        return 0;
    };
    auto copy = [&]() {
        const int left = copy_begin();
#pragma unroll
        for (int part = 0; part < T::PARTS; ++part) copy_part(left, part);
        copy_done();
    };

    // ---- products ----
    f32x4 acc[TI][TJ];
    float low = 1.0f;               // the least product of scales (0: sums that are not finite were met)
    // lane addresses of its operand rows (pieces g; pieces g + 4 lie 64 bytes on or back)
    const int xr = 16 * TJ * wt + l16, wr = 16 * TI * wc + tile_row<EXACT>(0, l16);
    const int xa = xr * BLOCK + 16 * (g ^ (l16 >> 1));
    const int wa = T::TOKENS * BLOCK + wr * BLOCK + 16 * (g ^ row_place<EXACT>(wr));

    // Operands are read from LDS ahead of their use: a column's x while the column before is multiplied, the next block's
    // first ones while this block's last column is.  So all of a block has been read, and its place is free, before
    // its last column, which is where the waves meet.
    uint4 wraw[TI][2], xraw[2][2];  // (as codes: an operand is made of them where it is used, not where it is read)
    float f[2], ws;
    auto read_w = [&](int at, int i) {
        // (where tile i's rows lie, further on by its first one, changes no bit that the placement reads)
        const char *p = codes[at] + tile_row<EXACT>(i, 0) * BLOCK;
        wraw[i][0] = *(const uint4 *)(p + wa);
        wraw[i][1] = *(const uint4 *)(p + (wa ^ 64));
    };
    auto read_x = [&](int at, int j) {
        const char *p = codes[at] + 16 * j * BLOCK;
        xraw[j & 1][0] = *(const uint4 *)(p + xa);
        xraw[j & 1][1] = *(const uint4 *)(p + (xa ^ 64));
        f[j & 1] = scales[at][16 * TJ * wt + 16 * j + l16];
        if (j == 0) ws = scales[at][T::TOKENS + 16 * TI * wc / BLOCK];
    };
    int used = 0, stored = 0;       // blocks that were waited for; of the waits to come, how many have a tile's stores before them
    // (the count of what is under way falls in the order of issue, loads and stores alike)
    constexpr int STORES = TJ * TI / (EXACT ? 1 : 2), LATER = T::COPIES * (STAGES - 2);
    static_assert(LATER + STORES < 64, "a wait counts to 63");
    // the next block is here (and what was read before is in registers)
    auto meet = [&]() {
        ++used;
        wait_copies<LATER, LATER + STORES>(__builtin_amdgcn_readfirstlane(copied - used < STAGES - 2 ? 0 : stored > 0 ? 2 : 1));
        --stored;
        __syncthreads();
    };
    auto multiply = [&](int at, int next, int left) {
        f32x4 part[3];
        float scale[2], wsb = ws;
        Operand<EXACT> w[TI], x;
        // a tile's sums are added while the products of the next two run
#pragma unroll
        for (int q = 0; q < TI * TJ + 2; ++q) {
            const int j = q / TI, i = q % TI;
            if (q < TI) w[i].set(wraw[i][0], wraw[i][1]);
            if (q < TI * TJ && i == 0) {
                scale[j & 1] = f[j & 1] * wsb;
                if (j & 1) low = fminf(fminf(low, fabsf(scale[0])), fabsf(scale[1]));
                x.set(xraw[j & 1][0], xraw[j & 1][1]);
                if (j + 1 < TJ) {
                    read_x(at, j + 1);
                } else {
                    meet();
                    read_x(next, 0);
                }
            }
            if (q < TI * TJ && i == 1 && j < T::PARTS) copy_part(left, j);
            if (q < TI * TJ) part[q % 3] = block_product(w[i], x);
            __builtin_amdgcn_sched_barrier(0);
            if (q < TI * TJ && j == TJ - 1) read_w(next, i);
            if (q > 1) {
                const int jw = (q - 2) / TI, iw = (q - 2) % TI;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[iw][jw][r] = fmaf(part[(q - 2) % 3][r], scale[jw & 1], acc[iw][jw][r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    };
    // A lane has runs of 8 (bf16) or 4 (fp32) neighbouring channels of TJ tokens.
    auto store = [&](const Place &tile) {
        const int c = tile.c0 + 16 * TI * wc;
#pragma unroll
        for (int j = 0; j < TJ; ++j) low = is(acc[0][j][0], NORMAL | DENORMAL | ZERO) ? low : 0.0f;
        if (tile.c0 + T::CHANNELS <= a.n && tile.t0 + T::TOKENS <= a.tokens) {
            float bias[TI][4];
#pragma unroll
            for (int i = 0; i < TI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) bias[i][r] = a.bias ? a.bias[c + tile_row<EXACT>(i, 4 * g) + r] : 0.0f;
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                char *at = a.out + (tile.t0 + 16 * (TJ * wt + j) + l16) * a.out_stride + (int64_t)c * (EXACT ? 4 : 2);
#pragma unroll
                for (int i = 0; i < TI; i += EXACT ? 1 : 2) {
                    float v[8];
#pragma unroll
                    for (int r = 0; r < (EXACT ? 4 : 8); ++r) v[r] = acc[i + r / 4][j][r % 4] + bias[i + r / 4][r % 4];
                    store_tok<!EXACT, EXACT ? 4 : 8>(at + tile_row<EXACT>(i, 4 * g) * (EXACT ? 4 : 2), v);
                }
            }
            stored = STAGES - 1;    // these STORES come after the copies of so many blocks
        } else {
#pragma unroll
            for (int j = 0; j < TJ; ++j)
#pragma unroll
                for (int i = 0; i < TI; ++i) store4(a, tile.t0 + 16 * (TJ * wt + j) + l16, c + tile_row<EXACT>(i, 4 * g), acc[i][j]);
            stored = 0;             // (their number is not known)
        }
    };

    int here = 0;                   // place in LDS of the block at hand
    bool sent = false;              // whether the copies that go with the block at hand were sent before
#pragma unroll
    for (int b = 0; b < STAGES - 1; ++b) copy();
    meet();
    read_x(0, 0);
#pragma unroll
    for (int i = 0; i < TI; ++i) read_w(0, i);
    for (int mine = blockIdx.x; mine < total; mine += gridDim.x) {
        const Place tile = place(mine);
        clear();
        for (int b = 0; b < a.blocks; ++b) {
            const int left = sent ? 0 : copy_begin();
            const int next = here + 1 == STAGES ? 0 : here + 1;
            multiply(here, next, left);             // (after the last block it reads what lies there, for nobody)
            if (!sent) copy_done();
            sent = false;
            here = next;
        }
        copy();                     // ahead of the outputs, which the next blocks then need not wait for
        sent = true;
        store(tile);
    }

    if (!__builtin_amdgcn_ballot_w64(is(low, ANY - NORMAL))) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // (before outputs are written again)
    const Anew n;
    const int m = n.lane & 15;
#pragma unroll 1
    for (int mine = blockIdx.x; mine < total; mine += gridDim.x) {
        const Place tile = place(mine);
        const int c = tile.c0 + 16 * TI * wc;
        bool again = false;
#pragma unroll 1
        for (int j = 0; j < TJ; ++j) again |= any_beyond(n, tile.t0 + 16 * (TJ * wt + j), c / BLOCK);
        if (!again) continue;
#pragma unroll 1
        for (int ij = 0; ij < TI * TJ; ++ij) {
            const int i = ij / TJ, t = tile.t0 + 16 * (TJ * wt + ij % TJ) + m;
            const f32x4 v = tile_apart<EXACT>(n, t, c + tile_row<EXACT>(i, m), c / BLOCK, 0, 1, n.a.blocks, n.a.blocks, f32x4{0, 0, 0, 0});
            store4(n.a, t, c + tile_row<EXACT>(i, 4 * (n.lane >> 4)), v);
        }
    }
}

// Workgroups: one for each CU, which takes tiles in turn.
template <bool EXACT, int WT, int WC, int TJ, int TI, int STAGES>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t st) {
    using T = Tile<WT, WC, TJ, TI, STAGES>;
    const int tiles_t = (a.tokens - 1) / T::TOKENS + 1, tiles_c = (a.n - 1) / T::CHANNELS + 1, total = tiles_t * tiles_c;
    const dim3 grid((unsigned)std::min(total, 256)), block(64 * T::WAVES);
    hipLaunchKernelGGL((product_kernel<EXACT, WT, WC, TJ, TI, STAGES>), grid, block, 0, st, a, tiles_t, tiles_c);
    return hipGetLastError();
}

// The tile whose rounds of 256 workgroups take the least time; a round's, for k = 4096, was measured (in 0.1 us).  192 tokens
// fill rounds that 128 and 256 do not: 1531 x 4096 -> 4096 fp32 54 us by 192 x 128 (256 tiles), 61 by 128 x 256, 73 by 128 x 128;
// 3000 x 4096 -> 4096 bf16 54 by 192 x 256, 59 by 256 x 256, 67 by 128 x 256.  The rule holds at other depths: with every tile
// tried at k = 128, 512, 1024 and 4096 on eight sizes from 512 x 2048 to 8192 x 12288 outputs in both types, it took the fastest
// or one within 5% of it.
template <bool EXACT>
hipError_t launch_many_tokens(const ProductArgs &a, hipStream_t st) {
    struct Choice {
        int tokens, channels, round;
    };
    constexpr Choice choices[] = {{64, 64, EXACT ? 222 : 150}, {64, 128, EXACT ? 295 : 195}, {128, 128, EXACT ? 412 : 270}, {192, 128, EXACT ? 552 : 358},
                                  {128, 256, EXACT ? 645 : 415}, {192, 256, EXACT ? 880 : 640}, {256, 256, 745}};
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < (EXACT ? 6 : 7); ++i) {
        const int64_t tiles = (int64_t)((a.tokens - 1) / choices[i].tokens + 1) * ((a.n - 1) / choices[i].channels + 1);
        const int64_t time = (tiles + 255) / 256 * choices[i].round;
        if (time <= least) best = i, least = time;
    }
    switch (best) {
        case 0: return launch_tiles<EXACT, 2, 2, 2, 2, 4>(a, st);
        case 1: return launch_tiles<EXACT, 2, 4, 2, 2, 3>(a, st);
        case 2: return launch_tiles<EXACT, 2, 4, 4, 2, 4>(a, st);
        case 3: return launch_tiles<EXACT, 2, 4, 6, 2, 3>(a, st);
        case 4: return launch_tiles<EXACT, 2, 4, 4, 4, 3>(a, st);
        case 5: return launch_tiles<EXACT, 2, 4, 6, 4, 2>(a, st);
        default: return launch_tiles<false, 2, 4, 8, 4, 2>(a, st);      // (bf16 only: twice the registers for fp32)
    }
}

// Few tokens, or too few tiles for half of the CUs, go without LDS: 128 x 4096 x 2048 (64 tiles) bf16 11.9 us, by tiles of 64 x 64
// 14.5, fp32 12.8 and 20.9; 256 x 4096 x 2048 (128) 15.8 and 14.6, fp32 16.9 and 21.1; 300 x 2048 x 2048 (160) 17.2 and 9.2, fp32
// 18.3 and 12.4.
template <bool EXACT>
hipError_t launch(const ProductArgs &a, hipStream_t st) {
    const int64_t tiles = (int64_t)((a.tokens - 1) / 64 + 1) * ((a.n - 1) / 64 + 1);
    return a.tokens <= 32 || tiles <= 128 ? launch_few_tokens<EXACT>(a, st) : launch_many_tokens<EXACT>(a, st);
}

}  // namespace

hipError_t launch_matmul(const lq_matmul &m, hipStream_t st) {
    if (m.tokens == 0) return hipSuccess;
    ProductArgs a;
    a.x = (const char *)m.x;
    a.w = (const char *)m.w;
    a.xs = m.x_scale;
    a.ws = m.w_scale;
    a.bias = m.bias;
    a.out = (char *)m.out;
    a.x_stride = row_bytes(m.tokens, m.x_stride, 1);
    a.xs_stride = row_bytes(m.tokens, m.x_scale_stride, 1);
    a.w_stride = row_bytes(m.n, m.w_stride, 1);
    a.out_stride = row_bytes(m.tokens, m.out_stride, m.out_dtype == LQ_TOKEN_BF16 ? 2 : 4);
    a.tokens = (int32_t)m.tokens;
    a.n = m.n;
    a.k = m.k;
    a.blocks = (m.k + BLOCK - 1) / BLOCK;
    a.out_bf16 = m.out_dtype == LQ_TOKEN_BF16;
    return a.out_bf16 ? launch<false>(a, st) : launch<true>(a, st);
}

}  // namespace lq
