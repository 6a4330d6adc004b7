// Selective state space scan, packed prompts and single tokens:
//   S_t = alpha_t S_{t-1} + delta_t k_t v_t^T,   o_t = S_t^T q_t + skip v_t,
// delta = softplus(dt + bias), alpha = exp(delta A), the state kept as S^T.
#include <algorithm>
#include <type_traits>

#include "lq_layer.hpp"
#include "lq_internal.hpp"

namespace lq {

namespace {

struct ScanArgs {
    const char *q, *k, *v, *dt;
    const float *A, *skip, *bias;
    char *o;
    char *state;
    const int32_t *cu, *slots;
    int32_t *err;
    int64_t tokens, q_stride, k_stride, v_stride, dt_stride, o_stride;    // strides in bytes
    int32_t batch, heads_v, group, n_slots, softplus, carry;
};

template <bool BF>
__device__ __forceinline__ void load8(const char *p, float *f) {
    unpack16<BF>(*(const uint4 *)p, f);
    if (!BF) unpack16<BF>(((const uint4 *)p)[1], f + 4);
}

// ---- single tokens ------------------------------------------------------------
//
// Bound: HBM, the state read and written once.  M rows of S^T per thread, 8 key
// channels each: 16 lanes hold a row, so the output's sum is a DPP row sum, and a
// workgroup holds 16 M rows, 8 / M workgroups a tile.  256 requests x 32 heads, fp32
// state: 188 us (5.8 TB/s) with one row a thread, 215 with eight.
template <bool BF, bool SBF, int M>
__global__ __launch_bounds__(NT) void scan_step_kernel(ScanArgs a) {
    constexpr int PARTS = 8 / M, SB = SBF ? 2 : 4;
    const int tid = threadIdx.x, l16 = tid & 15;
    const int tile = blockIdx.x / PARTS, r0 = (blockIdx.x % PARTS) * 16 * M + (tid >> 4);
    const int b = tile / a.heads_v, h = tile - b * a.heads_v;
    const int slot = state_row(a.state, a.slots, b, a.n_slots, a.err);
    float s[M][8];
    char *St = a.state + ((int64_t)slot * a.heads_v + h) * D * D * SB;
    const float fill = slot == BAD_SLOT ? nanf32() : 0.0f;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        if (slot >= 0) {
            load8<SBF>(St + ((r0 + 16 * m) * D + 8 * l16) * SB, s[m]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[m][j] = fill;
        }
    }
    const int64_t kc = ((int64_t)(h / a.group) * D + 8 * l16) * Tok<BF>::BYTES;
    float k[8], q[8], v[M];
    load8<BF>(a.k + (int64_t)b * a.k_stride + kc, k);
    load8<BF>(a.q + (int64_t)b * a.q_stride + kc, q);
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = load_tok<BF>(a.v + (int64_t)b * a.v_stride, (int64_t)h * D + r0 + 16 * m);
    const float bias = a.bias ? a.bias[h] : 0.0f, skip = a.skip ? a.skip[h] : 0.0f;
    const float delta = scan_delta(load_tok<BF>(a.dt + (int64_t)b * a.dt_stride, h) + bias, a.softplus);
    const float alpha = scan_alpha(delta * a.A[h]);
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] *= delta;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        float y = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[m][j] = fmaf(k[j], v[m], alpha * s[m][j]);
        if (SBF) {                                   // the output reads the state as it is stored
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t w = pk_bf16(s[m][j], s[m][j + 1]);
                s[m][j] = __uint_as_float(w << 16);
                s[m][j + 1] = __uint_as_float(w & 0xFFFF0000u);
            }
        }
        if (slot >= 0) store_tok<SBF, 8>(St + ((r0 + 16 * m) * D + 8 * l16) * SB, s[m]);
#pragma unroll
        for (int j = 0; j < 8; ++j) y = fmaf(s[m][j], q[j], y);
        y = row16_sum(y);
        if (a.skip) y = fmaf(skip, v[m], y);
        if (l16 == 0) {
            char *o = a.o + (int64_t)b * a.o_stride;
            if (BF) ((uint16_t *)o)[h * D + r0 + 16 * m] = (uint16_t)pk_bf16(y, y);
            else ((float *)o)[h * D + r0 + 16 * m] = y;
        }
    }
}

// ---- prompts --------------------------------------------------------------------
//
// A chunk of C tokens at a time, on the matrix cores.  With G_t the sum of the
// log decays from the chunk's start (base 2, fp64: differences of G are what
// counts, and one strong decay must not blur the weak ones after it),
//   o_t = 2^G_t S0^T q_t + sum_{j <= t} P_tj v_j + skip v_t,
//   P_tj = 2^(G_t - G_j) delta_j (q_t . k_j),
//   S   = 2^G_C S0 + sum_j k_j (w_j v_j)^T,   w_j = 2^(G_C - G_j) delta_j.
//
// One workgroup (4 waves) walks a segment of one head's tokens.  Wave w owns the
// value channels 32 w .. 32 w + 31 and all key channels of the state, which stays
// in registers as the accumulator of the last product.  An accumulator tile has
// its column in the lane and 4 rows in registers, an operand its outer index in
// the lane and 8 (bf16) or 1 (fp32) reduction slots; the sums may run in any
// order, so with rows and tokens dealt right a state tile, and a tile of P, is an
// operand as it stands and never goes through LDS.  Every wave computes P for
// itself (a tenth more products than sharing it out) and so waits for the others
// once a chunk, when the next chunk's rows have arrived: queries, keys and values
// are copied straight into LDS, one chunk ahead, token by token as they come, and
// the transposing LDS read turns them where a product sums over tokens.
//
// bf16 tokens are exact operands.  What is multiplied with them in fp32 (the
// state, P, w v) is split into three bf16 terms, which hold all its 24 bits: sums are
// those of fp32 also where they cancel.  (Two terms for the outputs are a tenth faster,
// 64 ragged prompts 180 instead of 203 us when the third came, but drop what lies below 2^-16 of a term.)
// fp32 tokens go through the fp32 matrix instructions.
//
// Bound: bf16, the issue of matrix and vector instructions, which do not overlap, beside
// HBM; fp32, the matrix cores (63% busy in the output pass).  64 ragged prompts, 16383
// tokens x 32 heads: 205 us; one of 32768 x 16 heads 259; 2048 fp32 tokens x 32 heads 99.

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum Mode {
    WHOLE = 0,      // one segment per sequence: state in, state out
    PARTS = 1,      // segments' own sums from zero, and their decays
    OUTPUT = 2      // outputs of segments whose start states are known
};

struct PromptArgs {
    ScanArgs s;
    float *parts;       // [segments][heads_v][D][D] (S^T): a segment's own sum, then its start state
    float *decays;      // [segments][heads_v]
    int32_t length;     // tokens of a segment
    int32_t segments;   // upper bound of their number (WHOLE: sequences)
    int32_t heads_k;
};

template <bool BF> struct Chunk {
    static constexpr int C = BF ? 32 : 16;          // tokens
    static constexpr int TILES = C / 16;
    static constexpr int PIECES = BF ? 16 : 32;     // 16-byte pieces of a row of q, k or v
    static constexpr int ROW = PIECES * 16;
    static constexpr int BYTES = C * ROW;           // 8 KiB either way
    static constexpr int GROUP = 4;                 // chunks whose steps and decays are prepared at once
    static constexpr int WAVES = GROUP * C / 64;    // ... by so many waves, the waves in turn
    typedef typename std::conditional<BF, bf16x8, f32x4>::type Operand;    // a piece of a row
    struct Rates {
        alignas(16) double g[C];                    // G_t
        alignas(16) float delta[C];
        alignas(16) float w[C];
    };
    // Place of a piece in its row: one piece of 16 rows lies in 16 different places
    // of a 256-byte line of banks, and so do the 4 pieces of 4 rows that a
    // transposing read (rows 4 r ..) or a column read of fp32 (rows r, r + 4, ..)
    // takes at once.  The counters show no conflicts for fp32, but 0.41 of the LDS's
    // active cycles for bf16, whose reads are not served in runs of 16 lanes; placements
    // with 64% fewer took the same time (64 ragged prompts x 32 heads 182-186 us, outputs from
    // two terms).
    __device__ static __forceinline__ int place(int row, int piece) {
        return piece ^ (BF ? 4 * (row & 3) + ((row >> 2) & 3) : row & 15);
    }
    // Offsets in an array's rows from which the products' operands follow by an exclusive
    // or: of piece g of row l16 (piece 4 s + g: s << 6), and, where a product sums over
    // tokens, of this lane's first columns of its first row (bf16 row 4 g + (l16 >> 2),
    // tile i: (i >> 1) << 6, and 8 for an odd i on top; fp32 row 4 g, row r and tile i:
    // r << 4 | i << 6, and r rows on top).
    __device__ static __forceinline__ int row_operand(int l16, int g) { return l16 * ROW + (place(l16, g) << 4); }
    __device__ static __forceinline__ int token_operand(int l16, int g) {
        return BF ? (4 * g + (l16 >> 2)) * ROW + (place(4 * g + (l16 >> 2), l16 & 3) << 4)
                  : 4 * g * ROW + (place(4 * g, l16 >> 2) << 4) + 4 * (l16 & 3);
    }
    // Key channel of register 0 of state tile i (0..7) in lane group g, and value
    // channel of a lane in tile u of its wave: bf16 deals rows so that tiles 2i and
    // 2i+1 hold 8 neighbouring key channels, and u = 0, 1 8 neighbouring outputs.
    __device__ static __forceinline__ int key_channel(int i, int g) {
        return BF ? 32 * (i >> 1) + 8 * g + 4 * (i & 1) : 16 * i + 4 * g;
    }
    __device__ static __forceinline__ int value_channel(int wave, int u, int l16) {
        return BF ? 32 * wave + 8 * (l16 >> 2) + 4 * u + (l16 & 3) : 32 * wave + 16 * u + l16;
    }
    // ... of output register 0 in tile u
    __device__ static __forceinline__ int out_channel(int wave, int u, int g) {
        return BF ? 32 * wave + 8 * g + 4 * u : 32 * wave + 16 * u + 4 * g;
    }
};

__device__ __forceinline__ bf16x8 pack8(const float *x) {
    const uint4 w = make_uint4(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]), pk_bf16(x[4], x[5]), pk_bf16(x[6], x[7]));
    return __builtin_bit_cast(bf16x8, w);
}
// Cuts 8 floats to bf16 and leaves in x what that dropped (exact).  Cut, not rounded:
// the upper half as it lies is the term (v_and at twice the rate of a shift, and one
// permutation packs two); two cut terms and a rounded one still hold 24 bits.
__device__ __forceinline__ bf16x8 split8(float *x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(x[2 * i]), b = __float_as_uint(x[2 * i + 1]);
        w[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        x[2 * i] -= __uint_as_float(a & 0xFFFF0000u);
        x[2 * i + 1] -= __uint_as_float(b & 0xFFFF0000u);
    }
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// LDS by its byte address.
template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) T *)(uintptr_t)at; }

__device__ __forceinline__ uint4 lds_read16(uint32_t at) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint4, lds_read<u32x4>(at));
}

// 8 rows x 16 columns of bf16 in LDS turned: the lanes of a 16-lane group pass the
// address of row l16 >> 2 of the first 4 rows, 4 columns each (the other 4 rows lie 16
// rows on), and a lane receives its column (number l16 & 3 of the 4 of lane l16 >> 2) of
// the 8 rows.
__device__ __forceinline__ bf16x8 frag_turned(uint32_t at) {
    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)at);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)(at + 16 * 256));
    const s16x8 r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, r);
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// 2^x with the rounding of a small exponent only (x rounded to fp32 as it is puts |x| ln 2
// half ulps on the result): for what a whole state is multiplied with.  (The weights of single
// tokens do without: where x is large, the weight is small beside the others.)  x = inf gives
// NaN.
__device__ __forceinline__ float exp2_wide(double x) {
    const double n = __builtin_rint(x);
    return ldexpf(exp2_hw((float)(x - n)), (int)n);
}

// Inclusive sums over each C = 16 or 32 lanes of a wave, and their totals.
template <int SHIFT>
__device__ __forceinline__ double row_shr_add(double x) {
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), 0x110 + SHIFT, 0xF, 0xF, true);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), 0x110 + SHIFT, 0xF, 0xF, true);
    return x + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double lane_value(double x, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane),
                            __builtin_amdgcn_readlane(__double2loint(x), lane));
}
template <int C>
__device__ __forceinline__ double scan_add_chunk(double x, int lane, double &all) {
    x = row_shr_add<1>(x);
    x = row_shr_add<2>(x);
    x = row_shr_add<4>(x);
    x = row_shr_add<8>(x);
    if (C == 16) {
        all = row_bcast<15>(x);
    } else {
        const double first = lane < 32 ? lane_value(x, 15) : lane_value(x, 47);
        if (lane & 16) x += first;
        all = lane < 32 ? lane_value(x, 31) : lane_value(x, 63);
    }
    return x;
}
__device__ __forceinline__ int scan_add32(int x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Segment `seg` of the packed sequences: its sequence (found[0]; -1: none) and its
// number within it (found[1]).  All 256 threads.
__device__ __forceinline__ void find_segment(const ScanArgs &a, int seg, int length, int *found, int *sums) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) found[0] = -1;
    int before = 0;
    for (int base = 0; base < a.batch; base += 256) {
        int n = 0;
        if (base + tid < a.batch) {
            const Span sp = sequence_span(a.cu, base + tid, a.tokens);
            n = (int)((sp.end - sp.begin + length - 1) / length);
        }
        const int inc = scan_add32(n, lane);
        if (lane == 63) sums[wave] = inc;
        __syncthreads();
        int off = before;
        for (int i = 0; i < wave; ++i) off += sums[i];
        if (seg >= off + inc - n && seg < off + inc) {
            found[0] = base + tid;
            found[1] = seg - (off + inc - n);
        }
        before += sums[0] + sums[1] + sums[2] + sums[3];
        __syncthreads();
        if (before > seg) break;
    }
}

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Whether what a wave's results that are not finite come from has NaN, but no infinity: its
// tokens' keys, values and queries, their steps, the state they started from.
template <bool BF, int MODE>
__device__ __forceinline__ bool only_nan(const ScanArgs &a, int64_t begin, int64_t end, int h, int wave, int lane,
                                         const float *state, bool given) {
    bool nan = false, inf = false;
    auto see = [&](float x) {
        nan |= x != x;
        inf |= fabsf(x) == INFINITY;
    };
    constexpr int V = Tok<BF>::V, PIECES = D / V;
    const int64_t piece = lane % PIECES * 16, key = (int64_t)(h / a.group) * D * Tok<BF>::BYTES + piece;
    const int64_t value = (int64_t)h * D * Tok<BF>::BYTES + piece;
#pragma unroll 4
    for (int64_t t = begin + lane / PIECES; t < end; t += 64 / PIECES) {
        float x[3][V];
        unpack16<BF>(*(const uint4 *)(a.k + t * a.k_stride + key), x[0]);
        unpack16<BF>(*(const uint4 *)(a.v + t * a.v_stride + value), x[1]);
        if (MODE != PARTS) unpack16<BF>(*(const uint4 *)(a.q + t * a.q_stride + key), x[2]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            see(x[0][i]);
            see(x[1][i]);
            if (MODE != PARTS) see(x[2][i]);
        }
    }
    const float bias = a.bias ? a.bias[h] : 0.0f;
    for (int64_t t = begin + lane; t < end; t += 64) see(scan_delta(load_tok<BF>(a.dt + t * a.dt_stride, h) + bias, a.softplus));
    see(a.A[h]);
    if (given)
        for (int i = lane; i < 32 * D; i += 64) see(state[32 * wave * D + i]);
    return __any(nan) && !__any(inf);
}

// The 32 value channels of wave `wave` of head h over tokens [begin, end) by the
// recurrence itself, token by token as scan_step does, from the state s (8 rows of S^T per
// lane: 32 wave + (lane >> 4) + 4 m, 8 key channels each).  Outputs and entries of the final
// state (NULL: not kept) are replaced where the stored ones are not finite.  For segments
// whose products met an infinity: a cut into terms leaves inf - inf there, a weight rounded
// to zero 0 inf, and neither is in the recurrence.  16 x 1024 tokens x 32 heads, the values
// of one token infinite: 1.7 ms instead of 0.17.  (Looked for in the
// operands, infinities would cost every chunk; the sum over results that finds them is within 1%.)
template <bool BF, int MODE>
__device__ __forceinline__ void walk_by_token(const ScanArgs &a, int64_t begin, int64_t end, int h, int wave, int lane,
                                              float (*s)[8], float *state) {
    const int l16 = lane & 15, r0 = 32 * wave + (lane >> 4);
    const float A = a.A[h], bias = a.bias ? a.bias[h] : 0.0f, skip = a.skip ? a.skip[h] : 0.0f;
    const int64_t kc = ((int64_t)(h / a.group) * D + 8 * l16) * Tok<BF>::BYTES;
#pragma unroll 1
    for (int64_t t = begin; t < end; ++t) {
        float k[8], q[8], v[8], was[8];
        char *o = a.o + t * a.o_stride;
        load8<BF>(a.k + t * a.k_stride + kc, k);
        if (MODE != PARTS) load8<BF>(a.q + t * a.q_stride + kc, q);
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            v[m] = load_tok<BF>(a.v + t * a.v_stride, (int64_t)h * D + r0 + 4 * m);
            if (MODE != PARTS) was[m] = load_tok<BF>(o, (int64_t)h * D + r0 + 4 * m);
        }
        const float delta = scan_delta(load_tok<BF>(a.dt + t * a.dt_stride, h) + bias, a.softplus);
        const float alpha = scan_alpha(delta * A);
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] *= delta;
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            const int64_t at = (int64_t)h * D + r0 + 4 * m;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[m][j] = fmaf(k[j], v[m], alpha * s[m][j]);
            if (MODE != PARTS) {
                float y = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) y = fmaf(s[m][j], q[j], y);
                y = row16_sum(y);
                if (a.skip) y = fmaf(skip, v[m], y);
                if (l16 == 0 && !is_finite(was[m])) {
                    if (BF) ((uint16_t *)o)[at] = (uint16_t)pk_bf16(y, y);
                    else ((float *)o)[at] = y;
                }
            }
        }
    }
    if (MODE == OUTPUT || !state) return;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
        float *row = state + (r0 + 4 * m) * D + 8 * l16;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!is_finite(row[j])) row[j] = s[m][j];
    }
}

template <bool BF, int MODE>
__global__ __launch_bounds__(256, !BF && MODE == PARTS ? 4 : 3) void scan_prompt_kernel(PromptArgs p) {
    using K = Chunk<BF>;
    constexpr int C = K::C, TILES = K::TILES;
    constexpr int ARRAYS = MODE == PARTS ? 2 : 3;           // keys, values, queries
    // (operands are addressed by exclusive ors within a row: it starts at a multiple of its size)
    __shared__ __attribute__((aligned(K::ROW))) char rows[2][ARRAYS][K::BYTES];
    __shared__ uint32_t steps[K::GROUP * C];                // dt of a group as it lies in memory
    __shared__ typename K::Rates rates[2][K::GROUP];
    const ScanArgs &a = p.s;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Workgroups go round the 8 XCDs: the heads that read one key head sit on one
    // of them, so its rows come from that XCD's L2.
    const int turn = blockIdx.x >> 3;
    const int kg = turn / a.group * 8 + (blockIdx.x & 7);
    if (kg >= p.segments * p.heads_k) return;
    const int seg = kg / p.heads_k, hk = kg - seg * p.heads_k;
    const int h = hk * a.group + turn % a.group;

    int b = seg;
    int64_t begin, end;
    if (MODE == WHOLE) {
        if (blockIdx.x == 0) check_seqlens(a.cu, a.batch, a.tokens, a.err, tid, 256);
        const Span sp = sequence_span(a.cu, b, a.tokens);
        begin = sp.begin;
        end = sp.end;
    } else {
        int *found = (int *)&rates[0][0];
        find_segment(a, seg, p.length, found, found + 2);
        b = __builtin_amdgcn_readfirstlane(found[0]);
        if (b < 0) return;
        const Span sp = sequence_span(a.cu, b, a.tokens);
        begin = sp.begin + (int64_t)__builtin_amdgcn_readfirstlane(found[1]) * p.length;
        end = min(begin + p.length, sp.end);
        __syncthreads();
    }

    // The rows of a chunk on their way into LDS, 2 KiB of each array per wave in two
    // copies: lane by lane the pieces that belong at the lane's place.  The second copy's
    // rows lie half a chunk on, their pieces `turned` bytes aside (bf16: the same pieces).
    constexpr int SECOND = C / 2;
    const int row0 = (64 * wave + lane) / K::PIECES;
    const int turned = 16 * (K::place(row0 + SECOND, lane % K::PIECES) - K::place(row0, lane % K::PIECES));
    const int64_t stride[3] = {a.k_stride, a.v_stride, a.q_stride};
    const char *from[ARRAYS];
    {
        const char *base[3] = {a.k + (int64_t)hk * K::ROW, a.v + (int64_t)h * K::ROW, a.q + (int64_t)hk * K::ROW};
#pragma unroll
        for (int n = 0; n < ARRAYS; ++n)
            from[n] = base[n] + (begin + row0) * stride[n] + 16 * K::place(row0, lane % K::PIECES);
    }
    auto copy_chunk = [&](int buf, int left) {            // left: tokens of the segment from this chunk on
#pragma unroll
        for (int n = 0; n < ARRAYS; ++n) {
            char *to = rows[buf][n] + 1024 * wave;
            if (left >= C) {
                dma16(from[n], lds_addr(to));
                dma16(from[n] + SECOND * stride[n] + turned, lds_addr(to + K::BYTES / 2));
            } else {
                // past the segment's end lie other tokens, or none: zeros stand in for them
                if (row0 < left) dma16(from[n], lds_addr(to));
                else *(uint4 *)(to + 16 * lane) = make_uint4(0u, 0u, 0u, 0u);
                if (row0 + SECOND < left) dma16(from[n] + SECOND * stride[n] + turned, lds_addr(to + K::BYTES / 2));
                else *(uint4 *)(to + K::BYTES / 2 + 16 * lane) = make_uint4(0u, 0u, 0u, 0u);
            }
            from[n] += C * stride[n];
        }
    };
    // Steps and decays of GROUP chunks' tokens, one per lane of WAVES waves: some 250
    // dependent instructions, so the waves take turns and are a group ahead.
    constexpr int GROUP_TOKENS = K::GROUP * C;
    const float A = a.A[h], bias = a.bias ? a.bias[h] : 0.0f;
    auto turn_of = [&](int group) { return wave / K::WAVES == group % (4 / K::WAVES); };
    auto own_token = [&] {                                // this lane's token of a group
        int again = lane;                                 // (not to be held in registers meanwhile)
        asm volatile("" : "+v"(again));
        return 64 * (wave % K::WAVES) + again;
    };
    auto copy_steps = [&](int64_t t0) {
        const int mine = own_token();
        if (t0 + mine < end)
            dma_element<Tok<BF>::BYTES>(a.dt + (t0 + mine) * a.dt_stride + h * Tok<BF>::BYTES,
                                        lds_addr(steps + 64 * (wave % K::WAVES)));
    };
    auto put_rates = [&](int group, int64_t t0) {
        const int mine = own_token();
        const bool there = t0 + mine < end;
        const float x = __uint_as_float(BF ? steps[mine] << 16 : steps[mine]);
        const float delta = there ? scan_delta(x + bias, a.softplus) : 0.0f;
        // (2^-1e5 is zero in any type; a bound keeps the sums exact beside it)
        double l = there ? (double)delta * (double)A * 1.4426950408889634074 : 0.0;
        l = l < -1e5 ? -1e5 : l;
        double all;
        const double G = scan_add_chunk<C>(l, lane, all);
        typename K::Rates &to = rates[group & 1][mine / C];
        to.g[mine % C] = G;
        to.delta[mine % C] = delta;
        to.w[mine % C] = exp2_hw((float)(all - G)) * delta;
    };

    if (begin < end) {
        if (turn_of(0)) copy_steps(begin);
        copy_chunk(0, (int)(end - begin));
    }

    // the state: tile [i][u], registers = 4 key channels
    f32x4 S[8][2];
    const int slot = MODE == WHOLE ? state_row(a.state, a.slots, b, a.n_slots, a.err) : NO_SLOT;
    float *Sp = MODE == WHOLE ? (float *)a.state + ((int64_t)slot * a.heads_v + h) * D * D
                              : p.parts + ((int64_t)seg * a.heads_v + h) * D * D;
    const bool given = MODE == OUTPUT || (MODE == WHOLE && slot >= 0 && a.carry);
    {
        const float fill = MODE == WHOLE && slot == BAD_SLOT ? nanf32() : 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float *row = Sp + K::value_channel(wave, u, l16) * D;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                S[i][u] = f32x4{fill, fill, fill, fill};
                if (given) S[i][u] = *(const f32x4 *)(row + K::key_channel(i, g));
            }
        }
    }
    const bool has_skip = MODE != PARTS && a.skip;
    const float skip = has_skip ? a.skip[h] : 0.0f;

    if (begin < end && turn_of(0)) {
        wait_vm_all();
        put_rates(0, begin);
    }
    double total = 0.0;                                   // log2 decay of the segment
    float odd_sum = 0.0f;                                 // NaN once a result is not finite
    int chunk = 0;
    for (int64_t t0 = begin; t0 < end; t0 += C, ++chunk) {
        // this chunk's rows have arrived, and nobody reads the last one's any more
        wait_vm_all();
        __syncthreads();
        const int buf = chunk & 1, group = chunk / K::GROUP;
        const typename K::Rates &rate = rates[group & 1][chunk % K::GROUP];
        // the next group: its steps set out with this one's first chunk and are there before its third
        if (turn_of(group + 1)) {
            if (chunk % K::GROUP == 0) copy_steps(t0 + GROUP_TOKENS);
            if (chunk % K::GROUP == 2) put_rates(group + 1, t0 + GROUP_TOKENS - 2 * C);
        }
        if (t0 + C < end) copy_chunk(buf ^ 1, (int)(end - t0) - C);

        // LDS addresses of the operands.  The empty asm keeps the compiler from holding the
        // dozens that follow from these two in registers of their own across the loop.
        uint32_t by_row = lds_addr(rows[buf][0]) + K::row_operand(l16, g);
        uint32_t by_token = lds_addr(rows[buf][0]) + K::token_operand(l16, g);
        asm volatile("" : "+v"(by_row), "+v"(by_token));
        constexpr uint32_t VALUES = K::BYTES, QUERIES = 2 * K::BYTES;
        typedef typename K::Operand Operand;

        f32x4 y[TILES][2], sc[TILES][TILES];
        if (MODE != PARTS) {
            // P^T's tiles (rows of keys J, columns of queries T, J <= T) and, from the same
            // queries, what the state gives: y^T = S^T q^T
#pragma unroll
            for (int T = 0; T < TILES; ++T) {
                y[T][0] = y[T][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int J = 0; J < TILES; ++J) sc[J][T] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int s = 0; s < (BF ? 4 : 8); ++s) {
                Operand kf[TILES], qf[TILES];
#pragma unroll
                for (int T = 0; T < TILES; ++T) {
                    kf[T] = lds_read<Operand>((by_row ^ (s << 6)) + 16 * T * K::ROW);
                    qf[T] = lds_read<Operand>((by_row ^ (s << 6)) + 16 * T * K::ROW + QUERIES);
                }
                if constexpr (BF) {
#pragma unroll
                    for (int T = 0; T < TILES; ++T)
#pragma unroll
                        for (int J = 0; J <= T; ++J) sc[J][T] = mfma(kf[J], qf[T], sc[J][T]);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = S[2 * s + (e >> 2)][u][e & 3];
                        const bf16x8 hi = split8(x), mid = split8(x), lo = pack8(x);
#pragma unroll
                        for (int T = 0; T < TILES; ++T) y[T][u] = mfma(hi, qf[T], y[T][u]);
#pragma unroll
                        for (int T = 0; T < TILES; ++T) y[T][u] = mfma(mid, qf[T], y[T][u]);
#pragma unroll
                        for (int T = 0; T < TILES; ++T) y[T][u] = mfma(lo, qf[T], y[T][u]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[0][0] = mfma(kf[0][e], qf[0][e], sc[0][0]);
                        y[0][0] = mfma(S[s][0][e], qf[0][e], y[0][0]);
                        y[0][1] = mfma(S[s][1][e], qf[0][e], y[0][1]);
                    }
                }
            }
            // 2^G_t on what the state gives, P's weights on the tiles
#pragma unroll
            for (int T = 0; T < TILES; ++T) {
                const double gt = rate.g[16 * T + l16];
                const float grown = exp2_wide(gt);
                y[T][0] *= grown;
                y[T][1] *= grown;
#pragma unroll
                for (int J = 0; J <= T; ++J) {
                    const int j0 = 16 * J + 4 * g;
                    const f32x4 dl = *(const f32x4 *)(rate.delta + j0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = sc[J][T][r] * (exp2_hw((float)(gt - rate.g[j0 + r])) * dl[r]);
                        sc[J][T][r] = J < T || 4 * g + r <= l16 ? x : 0.0f;
                    }
                }
            }
        }

        // Values as operands that sum over tokens, dealt like P's tiles: slots 4 J + r of
        // lane group g are the tokens 16 J + 4 g + r.
        bf16x8 xb[2];
        float xf[2][4];
        bool odd = false;                       // a value that is not finite
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (BF) {
                xb[u] = frag_turned((by_token ^ (wave << 6)) + VALUES + 8 * u);
                if (MODE != PARTS) {
                    const uint4 v = __builtin_bit_cast(uint4, xb[u]);
                    const uint32_t m = 0x7F807F80u, c = 0x00800080u;
                    odd |= ((((v.x & m) + c) | ((v.y & m) + c) | ((v.z & m) + c) | ((v.w & m) + c)) & 0x80008000u) != 0;
                }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    xf[u][r] = lds_read<float>((by_token ^ (r << 4 | (2 * wave + u) << 6)) + r * K::ROW + VALUES);
                    if (MODE != PARTS) odd |= (__float_as_uint(xf[u][r]) & 0x7F800000u) == 0x7F800000u;
                }
            }
        }

        if (MODE != PARTS) {
            if (!__any(odd)) {
                if constexpr (BF) {
#pragma unroll
                    for (int T = 0; T < 2; ++T) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = (e >> 2) <= T ? sc[e >> 2][T][e & 3] : 0.0f;
                        const bf16x8 hi = split8(x), mid = split8(x), lo = pack8(x);
#pragma unroll
                        for (int u = 0; u < 2; ++u) y[T][u] = mfma(xb[u], hi, y[T][u]);
#pragma unroll
                        for (int u = 0; u < 2; ++u) y[T][u] = mfma(xb[u], mid, y[T][u]);
#pragma unroll
                        for (int u = 0; u < 2; ++u) y[T][u] = mfma(xb[u], lo, y[T][u]);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        y[0][0] = mfma(xf[0][r], sc[0][0][r], y[0][0]);
                        y[0][1] = mfma(xf[1][r], sc[0][0][r], y[0][1]);
                    }
                }
            } else {
                // The products above multiply every value of the chunk, also by the zeros of
                // earlier tokens: with a value that is not finite, only what a token may see
                // is summed, value by value.
#pragma unroll
                for (int T = 0; T < TILES; ++T)
#pragma unroll
                    for (int J = 0; J <= T; ++J)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll 1
                            for (int from_g = 0; from_g < 4; ++from_g) {
                                const float pj = __shfl(sc[J][T][r], 16 * from_g + l16);
                                const int j = 16 * J + 4 * from_g + r;
#pragma unroll
                                for (int u = 0; u < 2; ++u)
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const int c = K::out_channel(wave, u, g) + e;
                                        const char *row = rows[buf][1] + j * K::ROW + (K::place(j, c / Tok<BF>::V) << 4);
                                        const float x = load_tok<BF>(row, c % Tok<BF>::V);
                                        if (j <= 16 * T + l16) y[T][u][e] = fmaf(pj, x, y[T][u][e]);
                                    }
                            }
            }
#pragma unroll
            for (int T = 0; T < TILES; ++T) {
                const int t = 16 * T + l16;
                float out[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] = y[T][e >> 2][e & 3];
                if (has_skip) {
                    float x[8];
                    if constexpr (BF) {
                        unpack16<true>(lds_read16((by_row ^ (wave << 6)) + 16 * T * K::ROW + VALUES), x);
                    } else {
                        unpack16<false>(lds_read16((by_row ^ (2 * wave << 6)) + VALUES), x);
                        unpack16<false>(lds_read16((by_row ^ ((2 * wave + 1) << 6)) + VALUES), x + 4);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[e] = fmaf(skip, x[e], out[e]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) odd_sum = fmaf(out[e], 0.0f, odd_sum);
                if (t0 + t < end) {
                    char *row = a.o + (t0 + t) * a.o_stride + (int64_t)h * K::ROW;
                    if constexpr (BF) {
                        store_tok<true, 8>(row + 2 * K::out_channel(wave, 0, g), out);
                    } else {
                        store_tok<false, 4>(row + 4 * K::out_channel(wave, 0, g), out);
                        store_tok<false, 4>(row + 4 * K::out_channel(wave, 1, g), out + 4);
                    }
                }
            }
        }

        // the state moves on
        if (MODE != OUTPUT || t0 + C < end) {
            const double g_end = rate.g[C - 1];
            const float keep = exp2_wide(g_end);
            if (MODE == PARTS) total += g_end;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                S[i][0] *= keep;
                S[i][1] *= keep;
            }
            if constexpr (BF) {
                bf16x8 wx[2][3];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float x[8];
                    unpack16<true>(__builtin_bit_cast(uint4, xb[u]), x);
#pragma unroll
                    for (int J = 0; J < 2; ++J) {
                        const f32x4 w = *(const f32x4 *)(rate.w + 16 * J + 4 * g);
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[4 * J + r] *= w[r];
                    }
                    wx[u][0] = split8(x);
                    wx[u][1] = split8(x);
                    wx[u][2] = pack8(x);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bf16x8 kf = frag_turned((by_token ^ ((i >> 1) << 6)) + 8 * (i & 1));
#pragma unroll
                    for (int term = 0; term < 3; ++term) {
                        S[i][0] = mfma(kf, wx[0][term], S[i][0]);
                        S[i][1] = mfma(kf, wx[1][term], S[i][1]);
                    }
                }
            } else {
                const f32x4 w = *(const f32x4 *)(rate.w + 4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x0 = xf[0][r] * w[r], x1 = xf[1][r] * w[r];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float kf = lds_read<float>((by_token ^ (r << 4 | i << 6)) + r * K::ROW);
                        S[i][0] = mfma(kf, x0, S[i][0]);
                        S[i][1] = mfma(kf, x1, S[i][1]);
                    }
                }
            }
        }
    }

    if (MODE != OUTPUT) {
        f32x4 sum[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};     // (eight chains, not one)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[u][r] = fmaf(S[i][u][r], 0.0f, sum[u][r]);
#pragma unroll
        for (int r = 0; r < 4; ++r) odd_sum += sum[0][r] + sum[1][r];
    }
    int again = lane;                           // (the first load's addresses would stay in registers all along)
    asm volatile("" : "+v"(again));
    const bool keeps = MODE == PARTS || (MODE == WHOLE && slot >= 0);
    // (a sequence that starts from NaN for want of a slot is NaN throughout, and NaN alone the
    // products carry on as the recurrence does)
    // What an infinity met is made again by the recurrence, whose arguments are read again
    // (none of them is held for this throughout the kernel).  A sequence that starts from NaN
    // for want of a slot is NaN throughout, and NaN alone the products carry on as it does.
    const PromptArgs *args = (const PromptArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    const bool walks = __any(odd_sum != odd_sum) && (MODE != WHOLE || slot != BAD_SLOT) &&
                       !only_nan<BF, MODE>(args->s, begin, end, h, wave, again, Sp, given);
    float start[8][8];
    if (walks) {
#pragma unroll
        for (int m = 0; m < 8; ++m) {
#pragma unroll
            for (int j = 0; j < 8; ++j) start[m][j] = 0.0f;
            if (given) load8<false>((const char *)(Sp + (32 * wave + (again >> 4) + 4 * m) * D + 8 * (again & 15)), start[m]);
        }
        wait_vm_all();
    }
    if (keeps) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float *row = Sp + K::value_channel(wave, u, again & 15) * D;
#pragma unroll
            for (int i = 0; i < 8; ++i) *(f32x4 *)(row + K::key_channel(i, again >> 4)) = S[i][u];
        }
    }
    if (walks) {
        wait_vm_all();                          // outputs and state are stored
        walk_by_token<BF, MODE>(args->s, begin, end, h, wave, again, start, keeps ? Sp : nullptr);
    }
    if (MODE == PARTS && tid == 0) p.decays[(int64_t)seg * a.heads_v + h] = exp2_wide(total > 1000.0 ? 1000.0 : total);
}

// Start states of the segments from their own sums, and the final state: per
// (sequence, head) a thread walks the segments with 4 entries of the state.
__global__ __launch_bounds__(256) void scan_join_kernel(PromptArgs p) {
    __shared__ int sums[4];
    const ScanArgs &a = p.s;
    const int tid = threadIdx.x;
    const int unit = blockIdx.x >> 4, at = ((blockIdx.x & 15) * 256 + tid) * 4;
    const int b = unit / a.heads_v, h = unit - b * a.heads_v;
    if (blockIdx.x == 0) check_seqlens(a.cu, a.batch, a.tokens, a.err, tid, 256);
    int first = 0;
    for (int i = tid; i < b; i += 256) {
        const Span sp = sequence_span(a.cu, i, a.tokens);
        first += (int)((sp.end - sp.begin + p.length - 1) / p.length);
    }
    first = __builtin_amdgcn_readlane(scan_add32(first, tid & 63), 63);
    if ((tid & 63) == 0) sums[tid >> 6] = first;
    __syncthreads();
    first = sums[0] + sums[1] + sums[2] + sums[3];
    const Span sp = sequence_span(a.cu, b, a.tokens);
    const int last = min(first + (int)((sp.end - sp.begin + p.length - 1) / p.length), p.segments);
    const int slot = state_row(a.state, a.slots, b, a.n_slots, a.err);
    float *St = (float *)a.state + ((int64_t)slot * a.heads_v + h) * D * D + at;
    f32x4 S = {0.0f, 0.0f, 0.0f, 0.0f};
    if (slot == BAD_SLOT) S = S + nanf32();
    else if (slot >= 0 && a.carry) S = *(const f32x4 *)St;
    const int64_t step = (int64_t)a.heads_v * D * D;
    float *part = p.parts + ((int64_t)first * a.heads_v + h) * D * D + at;
    const float *decay = p.decays + (int64_t)first * a.heads_v + h;
    for (int s = first; s < last; ++s, part += step, decay += a.heads_v) {
        const f32x4 own = *(const f32x4 *)part;
        *(f32x4 *)part = S;
        // (a decay is above zero however small: an infinity stays one where it is rounded to 0)
        const float by = *decay;
#pragma unroll
        for (int i = 0; i < 4; ++i) S[i] = (by == 0.0f && !is_finite(S[i]) ? S[i] : S[i] * by) + own[i];
    }
    if (slot >= 0) *(f32x4 *)St = S;
}

template <bool BF>
__global__ __launch_bounds__(256) void scan_gates_kernel(ScanArgs a, float *alpha, float *beta) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.tokens * a.heads_v) return;
    const int64_t t = i / a.heads_v;
    const int h = (int)(i - t * a.heads_v);
    const float delta = scan_delta(load_tok<BF>(a.dt + t * a.dt_stride, h) + (a.bias ? a.bias[h] : 0.0f), a.softplus);
    alpha[i] = scan_alpha(delta * a.A[h]);
    beta[i] = delta;
}

ScanArgs scan_args(const lq_dims &d, const lq_scan &s) {
    ScanArgs a;
    const int64_t es = s.dtype == LQ_TOKEN_BF16 ? 2 : 4;
    a.q = (const char *)s.q;
    a.k = (const char *)s.k;
    a.v = (const char *)s.v;
    a.dt = (const char *)s.dt;
    a.A = s.A;
    a.skip = s.skip;
    a.bias = s.dt_bias;
    a.o = (char *)s.o;
    a.state = (char *)s.state;
    a.cu = s.cu_seqlens;
    a.slots = s.slots;
    a.err = s.err;
    a.tokens = s.tokens;
    a.q_stride = row_bytes(s.tokens, s.q_stride, es);
    a.k_stride = row_bytes(s.tokens, s.k_stride, es);
    a.v_stride = row_bytes(s.tokens, s.v_stride, es);
    a.dt_stride = row_bytes(s.tokens, s.dt_stride, es);
    a.o_stride = row_bytes(s.tokens, s.o_stride, es);
    a.batch = d.batch;
    a.heads_v = d.heads_v;
    a.group = d.heads_v / d.heads_k;
    a.n_slots = s.n_slots;
    a.softplus = s.softplus;
    a.carry = s.carry;
    return a;
}

// How a prompt's work is split.  A sequence's chunks follow one another (2.9 us a chunk of
// 32 bf16 or 3.5 us of 16 fp32 tokens where a CU has one workgroup), so a launch has one
// workgroup per (sequence, head) unless the sequences are cut into segments, which costs a
// second pass over keys and values and the segments' states (64 KiB each, written, joined
// and read).  They are cut so that the launch has two workgroups per CU, and only where a
// segment is a small part of the longest sequence.  us without -> with, heads x tokens:
// bf16 16 x 512 50 -> 30, 16 x 320 33 -> 26, 16 x 256 (64 a segment) 28 -> 25, of four
// sequences 29 -> 33, 32 x 8192 729 -> 151; fp32 32 x 512 121 -> 53, 16 x 224 56 -> 40.
// Three workgroups' worth instead of two: 32 x 8192 147 instead of 151, 16 x 32768 260 instead
// of 259, fp32 32 x 2048 99 instead of 105; one: 158, 286, 107.
struct Split {
    int32_t length;         // tokens of a segment; 0: not cut
    int64_t segments;
    size_t bytes;
};
constexpr int64_t FULL = 512;                   // workgroups
size_t split_bytes(const lq_dims &d, int64_t segments) { return (size_t)segments * d.heads_v * (D * D + 4) * sizeof(float); }
int64_t least_chain(const lq_scan &s) { return s.dtype == LQ_TOKEN_BF16 ? 4 : 3; }      // segments, of the longest sequence

Split split_of(const lq_dims &d, const lq_scan &s) {
    Split r{0, d.batch, 0};
    const int64_t longest = s.max_len > 0 && s.max_len < s.tokens ? s.max_len : s.tokens;
    if ((int64_t)d.batch * d.heads_v >= FULL) return r;
    const int64_t length = std::max<int64_t>((s.tokens * d.heads_v / FULL + 63) / 64 * 64, 64);
    if (longest <= least_chain(s) * length) return r;
    r.length = (int32_t)length;
    r.segments = s.tokens / length + d.batch;   // each sequence's last segment may be short
    r.bytes = split_bytes(d, r.segments);
    return r;
}

// The most that split_of gives for up to s.tokens tokens and any max_len.  A segment's length
// is rounded up to 64, so their number falls each time a longer one is taken: it is largest
// for the most tokens that the shortest length, 64, serves; where those are not cut, no
// others are.
size_t most_split_bytes(const lq_dims &d, const lq_scan &s) {
    if ((int64_t)d.batch * d.heads_v >= FULL) return 0;
    const int64_t tokens = std::min(s.tokens, (65 * FULL - 1) / d.heads_v);
    return tokens > least_chain(s) * 64 ? split_bytes(d, tokens / 64 + d.batch) : 0;
}

template <bool BF>
hipError_t launch_prompt(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    const Split sp = split_of(d, s);
    PromptArgs p;
    p.s = scan_args(d, s);
    p.heads_k = d.heads_k;
    p.length = sp.length;
    p.segments = (int32_t)sp.segments;
    p.parts = (float *)s.workspace;
    p.decays = sp.length ? p.parts + sp.segments * d.heads_v * D * D : nullptr;      // (not cut: no workspace)
    const int64_t groups = (sp.segments * d.heads_k + 7) / 8 * 8;
    const dim3 grid((unsigned)(groups * p.s.group));
    if (!sp.length) {
        hipLaunchKernelGGL((scan_prompt_kernel<BF, WHOLE>), grid, dim3(256), 0, st, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((scan_prompt_kernel<BF, PARTS>), grid, dim3(256), 0, st, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(scan_join_kernel, dim3(16 * d.batch * d.heads_v), dim3(256), 0, st, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((scan_prompt_kernel<BF, OUTPUT>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

template <bool BF, bool SBF>
hipError_t launch_step(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    const ScanArgs a = scan_args(d, s);
    const int tiles = d.batch * d.heads_v;
    // Rows per thread, us a call (1, 2, 4, 8): fp32 8192 tiles 186, 201, 206, 215; 2048 49, 51,
    // 53, 58; 512 14.5, 13.0, 13.4, 13.7; bf16 8192 123, 101, 104, 115; 16 4.2, 4.2, 4.6, 5.0.
    if constexpr (!SBF) {
        if (tiles >= 2048) {
            hipLaunchKernelGGL((scan_step_kernel<BF, SBF, 1>), dim3(8 * tiles), dim3(NT), 0, st, a);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((scan_step_kernel<BF, SBF, 2>), dim3(4 * tiles), dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t scan_workspace_bytes(const lq_dims &d, const lq_scan &s) {
    return s.max_len > 0 ? split_of(d, s).bytes : most_split_bytes(d, s);
}

hipError_t launch_scan_prompt(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    return s.dtype == LQ_TOKEN_BF16 ? launch_prompt<true>(d, s, st) : launch_prompt<false>(d, s, st);
}

hipError_t launch_scan_step(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    const bool sbf = s.state_dtype == LQ_STATE_BF16;
    if (s.dtype == LQ_TOKEN_BF16) return sbf ? launch_step<true, true>(d, s, st) : launch_step<true, false>(d, s, st);
    return sbf ? launch_step<false, true>(d, s, st) : launch_step<false, false>(d, s, st);
}

hipError_t launch_scan_gates(const lq_dims &d, const lq_scan &s, float *alpha, float *beta, hipStream_t st) {
    const ScanArgs a = scan_args(d, s);
    const int64_t n = a.tokens * a.heads_v;
    if (n == 0) return hipSuccess;
    const dim3 grid((unsigned)((n + 255) / 256));
    if (s.dtype == LQ_TOKEN_BF16) hipLaunchKernelGGL((scan_gates_kernel<true>), grid, dim3(256), 0, st, a, alpha, beta);
    else hipLaunchKernelGGL((scan_gates_kernel<false>), grid, dim3(256), 0, st, a, alpha, beta);
    return hipGetLastError();
}

}  // namespace lq
