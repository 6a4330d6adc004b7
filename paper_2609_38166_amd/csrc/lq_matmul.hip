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
// Bound: HBM, the weight.  A workgroup owns 16 CT channels of 16 TT tokens; its waves take the blocks of k in turn, AHEAD
// of them at a time, straight from memory into registers, and join their sums in LDS.
template <bool EXACT, int TT, int CT, int WAVES, int AHEAD>
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
    struct Pieces {
        uint4 w[CT][2], x[TT][2];
        float ws[CT], s[TT];
    };
    // block b's pieces; past k (the end of a last block that is shorter) zeros
    auto load = [&](Pieces &o, int b, bool whole) {
        const int at = b * BLOCK + 16 * g;
        auto pieces = [&](const char *row, uint4 *p) {
            const uint4 none = make_uint4(0, 0, 0, 0);
            p[0] = whole || at < a.k ? *(const uint4 *)(row + at) : none;
            p[1] = whole || at + 64 < a.k ? *(const uint4 *)(row + at + 64) : none;
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
        Operand<EXACT> w[CT];
#pragma unroll
        for (int i = 0; i < CT; ++i) w[i].set(o.w[i][0], o.w[i][1]);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            Operand<EXACT> x;
            x.set(o.x[j][0], o.x[j][1]);
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const f32x4 p = block_product(w[i], x);
                const float f = o.s[j] * o.ws[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], f, acc[i][j][r]);
            }
        }
    };
    const int whole = a.k / BLOCK;
    int b = wave;
    for (; b + (AHEAD - 1) * WAVES < whole; b += AHEAD * WAVES) {
        Pieces o[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(o[u], b + u * WAVES, true);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) add(o[u]);
    }
    for (; b < a.blocks; b += WAVES) {
        Pieces o;
        load(o, b, b < whole);
        add(o);
    }
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) parts[wave][i * TT + j][lane] = acc[i][j];
    __syncthreads();
    for (int e = tid; e < TT * CT * 64; e += 64 * WAVES) {
        const int tile = e >> 6, from = e & 63;
        f32x4 v = parts[0][tile][from];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += parts[i][tile][from];
        store4(a, t0 + 16 * (tile % TT) + (from & 15), c0 + 16 * (tile / TT) + 4 * (from >> 4), v);
    }
}

template <int TT, int CT, int WAVES, int AHEAD>
hipError_t launch_few(const ProductArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)((a.n - 1) / (16 * CT) + 1), (unsigned)((a.tokens - 1) / (16 * TT) + 1)), block(64 * WAVES);
    if (a.out_bf16) hipLaunchKernelGGL((product_few_kernel<false, TT, CT, WAVES, AHEAD>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((product_few_kernel<true, TT, CT, WAVES, AHEAD>), grid, block, 0, st, a);
    return hipGetLastError();
}

// ---- many tokens ------------------------------------------------------------------
//
// Bound: the matrix cores, with the LDS beside them.  A workgroup owns a tile of 16 WT TJ tokens x 16 WC TI channels, a wave
// TJ x TI tiles of 16 x 16, all sums in registers.  Blocks of k are copied straight into LDS, STAGES - 1 ahead; a row's 8
// pieces are placed by an exclusive or with bits of the row, so that the 16 rows that a read takes at once lie in 16 different
// places of a 256-byte line of banks.  Channels are dealt to a wave's tiles so that a lane ends up with 16 bytes of
// neighbouring outputs of a token at a time, and 4 lanes with 64.
__device__ const uint4 no_codes = {0, 0, 0, 0};

// Copies into LDS as dma16's and dma_element's: 16 bytes per lane from a uniform base and a lane's offset, and one element.
// Nothing is copied where `left` is not positive: no lane is on then (all are where these are called).  By the mask and
// not by a branch, so that the products around them stay one run of instructions.
__device__ __forceinline__ void dma16_if(int left, uint64_t base, uint32_t offset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_cmp_gt_i32 %3, 0\n\ts_cselect_b64 exec, -1, 0\n\t"
                 "global_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" :: "v"(offset), "s"(base), "s"(lds_base), "s"(left) : "memory", "scc");
}
__device__ __forceinline__ void dma4_if(int left, const void *g, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_cmp_gt_i32 %2, 0\n\ts_cselect_b64 exec, -1, 0\n\t"
                 "global_load_lds_dword %0, off\n\ts_mov_b64 exec, -1" :: "v"(g), "s"(lds_base), "s"(left) : "memory", "scc");
}
// Waits until at most N copies are under way, or none where `more` is negative.
template <int N>
__device__ __forceinline__ void wait_copies(int more) {
    if (N == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else asm volatile("s_cmp_ge_i32 %1, 0\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(0)\n1:\n\ts_waitcnt vmcnt(%0)" :: "n"(N), "s"(more) : "memory", "scc");
}

template <int WT, int WC, int TJ, int TI, int STAGES>
struct Tile {
    static constexpr int WAVES = WT * WC, TOKENS = 16 * WT * TJ, CHANNELS = 16 * WC * TI;
    static constexpr int X_COPIES = TOKENS / 8 / WAVES, W_COPIES = CHANNELS / 8 / WAVES;   // of 8 rows, per wave
    static constexpr int COPIES = X_COPIES + W_COPIES + 1;                                 // ... and one of scales
    static constexpr int STAGE = (TOKENS + CHANNELS) * BLOCK;
    static_assert(TOKENS % (8 * WAVES) == 0 && CHANNELS % (8 * WAVES) == 0 && TOKENS % 64 == 0, "whole copies");
    static_assert(TJ % 2 == 0 && TI % 2 == 0, "columns take turns in two registers, tiles of bf16 outputs go in pairs");
};

// Row m of a wave's tile i among its 16 TI rows of w, and the bits that place a row's pieces: they differ for the 8 pairs of
// rows of a tile.
template <bool EXACT>
__device__ __forceinline__ int tile_row(int i, int m) { return EXACT ? 16 * i + m : 32 * (i >> 1) + 8 * (m >> 2) + 4 * (i & 1) + (m & 3); }
template <bool EXACT>
__device__ __forceinline__ int row_place(int row) { return EXACT ? row >> 1 & 7 : (row >> 3 & 3) | (row >> 1 & 1) << 2; }

template <bool EXACT, int WT, int WC, int TJ, int TI, int STAGES>
__global__ __launch_bounds__(64 * WT * WC) void product_kernel(ProductArgs a, int tiles_t, int tiles_c) {
    using T = Tile<WT, WC, TJ, TI, STAGES>;
    __shared__ __attribute__((aligned(1024))) char codes[STAGES][T::STAGE];     // rows of x, then of w
    __shared__ float scales[STAGES][T::TOKENS];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / WC, wc = wave % WC;

    // Workgroups go round the 8 XCDs: each gets neighbouring tiles, GROUP of tokens side by side, whose rows its L2 shares.
    constexpr int GROUP = 4;
    const int total = tiles_t * tiles_c, per = total / 8, more = total % 8, xcd = blockIdx.x % 8;
    const int id = xcd * per + min(xcd, more) + blockIdx.x / 8;
    const int band = id / (GROUP * tiles_c), first = band * GROUP, high = min(GROUP, tiles_t - first);
    const int in_band = id - band * GROUP * tiles_c;
    const int t0 = (first + in_band % high) * T::TOKENS, c0 = in_band / high * T::CHANNELS;

    // this lane's rows and pieces in the copies
    const int row8 = lane >> 3, slot = lane & 7;
    uint32_t xo[T::X_COPIES], wo[T::W_COPIES];
    int xp[T::X_COPIES], wp[T::W_COPIES];
#pragma unroll
    for (int i = 0; i < T::X_COPIES; ++i) {
        const int row = 8 * (wave * T::X_COPIES + i) + row8;
        xp[i] = 16 * (slot ^ (row >> 1 & 7));
        xo[i] = (uint32_t)(min(row, a.tokens - 1 - t0) * a.x_stride) + xp[i];
    }
#pragma unroll
    for (int i = 0; i < T::W_COPIES; ++i) {
        const int row = 8 * (wave * T::W_COPIES + i) + row8;
        wp[i] = 16 * (slot ^ row_place<EXACT>(row));
        wo[i] = (uint32_t)(min(row, a.n - 1 - c0) * a.w_stride) + wp[i];
    }
    const uint64_t xbase = (uint64_t)(a.x + t0 * a.x_stride), wbase = (uint64_t)(a.w + c0 * a.w_stride);
    const int scale_part = wave % (T::TOKENS / 64);
    const float *scale_row = a.xs + min(t0 + 64 * scale_part + lane, a.tokens - 1) * a.xs_stride;
    const int whole = a.k / BLOCK;

    // whole block b on its way (not if there is none)
    auto copy = [&](int b) {
        const int st = b % STAGES;
        const uint32_t xl = lds_addr(codes[st]) + wave * T::X_COPIES * 1024;
        const uint32_t wl = lds_addr(codes[st]) + T::TOKENS * BLOCK + wave * T::W_COPIES * 1024;
        const uint64_t at = (uint64_t)b * BLOCK;
        const int left = whole - b;
#pragma unroll
        for (int i = 0; i < T::X_COPIES; ++i) dma16_if(left, xbase + at, xo[i], xl + 1024 * i);
#pragma unroll
        for (int i = 0; i < T::W_COPIES; ++i) dma16_if(left, wbase + at, wo[i], wl + 1024 * i);
        dma4_if(left, scale_row + b, lds_addr(scales[st]) + 256 * scale_part);
    };

    f32x4 acc[TI][TJ] = {};
    // lane addresses of its operand rows (pieces g; pieces g + 4 lie 64 bytes on or back)
    const int xr = 16 * TJ * wt + l16, wr = 16 * TI * wc + tile_row<EXACT>(0, l16);
    const int xa = xr * BLOCK + 16 * (g ^ (l16 >> 1));
    const int wa = T::TOKENS * BLOCK + wr * BLOCK + 16 * (g ^ row_place<EXACT>(wr));
    const float *ws_row = a.ws + (int64_t)(min(c0 + 16 * TI * wc, a.n - 1) / BLOCK) * a.blocks;
    float ws_lane = 0.0f;                           // the weight's scales of 64 blocks, one a lane

    // Operands are read from LDS ahead of their use: a column's x while the column before is multiplied, the next block's
    // first ones while this block's last column is.  So all of a block has been read, and its place is free, before
    // its last column, which is where the waves meet and the next copies are sent.
    Operand<EXACT> w[TI], x[2];
    float f[2];
    auto read_w = [&](int b, int i) {
        // (where tile i's rows lie, further on by its first one, changes no bit that the placement reads)
        const char *p = codes[b % STAGES] + tile_row<EXACT>(i, 0) * BLOCK;
        w[i].set(*(const uint4 *)(p + wa), *(const uint4 *)(p + (wa ^ 64)));
    };
    auto read_x = [&](int b, int j) {
        const char *p = codes[b % STAGES] + 16 * j * BLOCK;
        x[j & 1].set(*(const uint4 *)(p + xa), *(const uint4 *)(p + (xa ^ 64)));
        f[j & 1] = scales[b % STAGES][16 * TJ * wt + 16 * j + l16];
    };
    // (what was read before is in registers when the waves meet)
    auto meet = [&](int b) {
        wait_copies<T::COPIES *(STAGES - 2)>(whole + 1 - STAGES - b);
        __syncthreads();
    };
    auto multiply = [&](int b, bool ahead) {
        if ((b & 63) == 0) {
            ws_lane = ws_row[min(b + lane, a.blocks - 1)];
            asm volatile("" : "+v"(ws_lane));       // (its wait belongs here, not into every block)
        }
        const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ws_lane), b & 63));
        f32x4 part[3];
        float scale[2];
        // a tile's sums are added while the products of the next two run
#pragma unroll
        for (int q = 0; q < TI * TJ + 2; ++q) {
            const int j = q / TI, i = q % TI;
            if (q < TI * TJ && i == 0) {
                scale[j & 1] = f[j & 1] * ws;
                if (j + 1 < TJ) {
                    read_x(b, j + 1);
                } else if (ahead) {
                    meet(b + 1);
                    copy(b + STAGES);
                    read_x(b + 1, 0);
                }
            }
            if (q < TI * TJ) part[q % 3] = block_product(w[i], x[j & 1]);
            __builtin_amdgcn_sched_barrier(0);
            if (ahead && q < TI * TJ && j == TJ - 1) read_w(b + 1, i);
            if (q > 1) {
                const int jw = (q - 2) / TI, iw = (q - 2) % TI;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[iw][jw][r] = fmaf(part[(q - 2) % 3][r], scale[jw & 1], acc[iw][jw][r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto begin = [&](int b) {
        read_x(b, 0);
#pragma unroll
        for (int i = 0; i < TI; ++i) read_w(b, i);
    };
    if (whole > 0) {
#pragma unroll
        for (int b = 0; b < STAGES - 1; ++b) copy(b);
        meet(0);
        copy(STAGES - 1);
        begin(0);
        // (after the last one it reads what lies there, for nobody)
        for (int b = 0; b < whole; ++b) multiply(b, true);
    }
    if (whole < a.blocks) {                         // a last block that is shorter: zeros past k
        const int left = a.k - whole * BLOCK, st = whole % STAGES;
        const uint32_t xl = lds_addr(codes[st]) + wave * T::X_COPIES * 1024;
        const uint32_t wl = lds_addr(codes[st]) + T::TOKENS * BLOCK + wave * T::W_COPIES * 1024;
        const char *none = (const char *)&no_codes, *x0 = (const char *)xbase + whole * BLOCK, *w0 = (const char *)wbase + whole * BLOCK;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < T::X_COPIES; ++i) dma16(xp[i] < left ? x0 + xo[i] : none, xl + 1024 * i);
#pragma unroll
        for (int i = 0; i < T::W_COPIES; ++i) dma16(wp[i] < left ? w0 + wo[i] : none, wl + 1024 * i);
        dma_element<4>(scale_row + whole, lds_addr(scales[st]) + 256 * scale_part);
        wait_vm_all();
        __syncthreads();
        begin(whole);
        multiply(whole, false);
    }
    // A lane has runs of 8 (bf16) or 4 (fp32) neighbouring channels of TJ tokens.
    const int c = c0 + 16 * TI * wc;
    if (c0 + T::CHANNELS <= a.n) {
        float bias[TI][4];
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) bias[i][r] = a.bias ? a.bias[c + tile_row<EXACT>(i, 4 * g) + r] : 0.0f;
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const int t = t0 + 16 * (TJ * wt + j) + l16;
            char *at = a.out + t * a.out_stride + (int64_t)c * (EXACT ? 4 : 2);
            if (t >= a.tokens) continue;
#pragma unroll
            for (int i = 0; i < TI; i += EXACT ? 1 : 2) {
                float v[8];
#pragma unroll
                for (int r = 0; r < (EXACT ? 4 : 8); ++r) v[r] = acc[i + r / 4][j][r % 4] + bias[i + r / 4][r % 4];
                store_tok<!EXACT, EXACT ? 4 : 8>(at + tile_row<EXACT>(i, 4 * g) * (EXACT ? 4 : 2), v);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int i = 0; i < TI; ++i) store4(a, t0 + 16 * (TJ * wt + j) + l16, c + tile_row<EXACT>(i, 4 * g), acc[i][j]);
    }
}

template <bool EXACT, int WT, int WC, int TJ, int TI, int STAGES>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t st) {
    using T = Tile<WT, WC, TJ, TI, STAGES>;
    const int tiles_t = (a.tokens - 1) / T::TOKENS + 1, tiles_c = (a.n - 1) / T::CHANNELS + 1;
    const dim3 grid((unsigned)(tiles_t * tiles_c)), block(64 * T::WAVES);
    hipLaunchKernelGGL((product_kernel<EXACT, WT, WC, TJ, TI, STAGES>), grid, block, 0, st, a, tiles_t, tiles_c);
    return hipGetLastError();
}

}  // namespace

size_t matmul_workspace_bytes(const lq_matmul &) { return 0; }

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
    if (m.tokens <= 16) return launch_few<1, 1, 8, 4>(a, st);
    const int64_t large = (int64_t)((a.tokens - 1) / 256 + 1) * ((a.n - 1) / 256 + 1);
    if (large >= 200) return a.out_bf16 ? launch_tiles<false, 2, 4, 8, 4, 2>(a, st) : launch_tiles<true, 2, 4, 8, 2, 3>(a, st);
    if (m.tokens > 64) return a.out_bf16 ? launch_tiles<false, 2, 2, 4, 4, 4>(a, st) : launch_tiles<true, 2, 2, 4, 4, 4>(a, st);
    return launch_few<4, 4, 4, 1>(a, st);
}

}  // namespace lq
