// Rows on their way into a product: the residual's addition and the norm of hidden rows, the norm and the gate of a layer's
// outputs, and weights, in the token types or in E4M3 with a scale for each block of 128.
//   add_norm   h = x + residual,  y = h / sqrt(mean h^2 + eps) w
//   gate_norm  y = x / sqrt(mean x^2 + eps) w act(gate), or the norm of x act(gate)
//
// Bound: HBM; the gated norm's instructions come near it.  A lane owns 8 channels, so that a block of 128 is a row of 16 lanes
// (its largest magnitude by DPP); a row of channels stays in the registers of 8 to 1024 lanes between its sum of squares and
// its output.  bf16 to E4M3: add_norm of 8192 x 4096 48 us (4.9 TB/s), gate_norm of 8192 x 32 heads of 128 37-38 (4.5 TB/s; 290
// vector instructions for 8 values a lane, 370 took 49-50); the gate first, a weight per head and heads of 64 to 8192 37-40.  Lengths
// that leave lanes idle or need workgroups of 1024 are further off: 8192 x 11 heads of 384 47 us, of 37 by their bytes, 2048 rows of
// 16384 48, of 36.
#include <algorithm>

#include "lq_e4m3.hpp"
#include "lq_internal.hpp"

namespace lq {

namespace {

struct RowArgs {
    const char *x, *second;         // second: the residual (may be null) or the gate
    const float *weight;            // may be null
    char *sum, *out;                // sum: residual_out (may be null)
    float *scale;
    int64_t x_stride, second_stride, sum_stride, out_stride;    // bytes
    int64_t scale_stride;           // floats
    uint32_t tokens, heads, heads_turn;     // rows: heads_turn a token, those past heads are none
    uint32_t step;                  // a group of lanes takes every step-th token
    int32_t length, norm, out_type, act, first, weight_heads;
    float eps;
};

// 8 values as they lie in memory
template <bool BF> struct Raw {
    uint4 p[BF ? 1 : 2];
    __device__ __forceinline__ void load(const char *at) {
        p[0] = *(const uint4 *)at;
        if (!BF) p[BF ? 0 : 1] = ((const uint4 *)at)[1];
    }
    __device__ __forceinline__ void values(float *f) const {
        unpack16<BF>(p[0], f);
        if (!BF) unpack16<BF>(p[BF ? 0 : 1], f + 4);
    }
};

// Sum over the L lanes (8 .. 64 neighbours, or the workgroup) of a row.
template <int L>
__device__ __forceinline__ float row_sum(float x, float *sums) {
    x += dpp<DPP_XOR1>(x);
    x += dpp<DPP_XOR2>(x);
    if (L == 8) return x + dpp<DPP_HALF_MIRROR>(x);
    x += dpp<DPP_ROR4>(x);
    x += dpp<DPP_ROR8>(x);
    if (L >= 32) x += __shfl_xor(x, 16);
    if (L >= 64) x += __shfl_xor(x, 32);
    if (L > 64) {
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0f;
#pragma unroll
        for (int i = 0; i < L / 64; ++i) x += sums[i];
        __syncthreads();
    }
    return x;
}

// sigmoid(z) = 1 / (1 + e), or e / (1 + e) for z < 0, of e = exp(-|z|): the hardware's exponential of the rounded product with
// log2(e), times 1 + what the rounding left (so a large |z| keeps its bits), and the hardware's reciprocal, 1 ulp each.  The
// kernel is bound by such instructions: with expf and an IEEE division 8192 x 32 heads of 128 took 52 us.  (NaN gives
// any number: see gate_values.)
__device__ __forceinline__ float sigmoid(float z) {
    const float a = fminf(fabsf(z), 150.0f);
    const float t = -1.44269502f * a, rest = fmaf(a, -1.92596303e-8f, fmaf(a, -1.44269502f, -t));
    const float e0 = __builtin_amdgcn_exp2f(t), e = fmaf(e0 * rest, 0.693147181f, e0);
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    return z < 0.0f ? e * r : r;
}
__device__ __forceinline__ void gate_values(float *z, int act) {
    if (act == LQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= sigmoid(z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = z[i] != z[i] ? z[i] : sigmoid(z[i]);
    }
}

// A group of L lanes keeps its head (heads of the next tokens follow a constant distance on) and takes tokens in turn.
template <int L, int P, bool XB, bool SB, bool GATE>
__global__ __launch_bounds__(L > 256 ? L : 256) void rows_kernel(RowArgs a) {
    constexpr int THREADS = L > 256 ? L : 256, PER = THREADS / L;
    __shared__ float sums[L > 64 ? L / 64 : 1];
    const int l = threadIdx.x % L, l16 = threadIdx.x & 15;
    const uint32_t row = blockIdx.x * PER + threadIdx.x / L;
    uint32_t t = GATE ? row / a.heads_turn : row;
    const uint32_t h = GATE ? row - t * a.heads_turn : 0;
    const int64_t col = GATE ? (int64_t)h * a.length : 0;
    const bool there = !GATE || h < a.heads;        // (the lanes of a head that is none take part in the exchanges)
    if (t >= a.step) return;                        // (groups past step * heads_turn: whole pairs of heads)
    float w[P][8];
    bool in[P];
#pragma unroll
    for (int p = 0; p < P; ++p) in[p] = there && 8 * (p * L + l) < a.length;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[p][i] = 1.0f;
        if (a.weight && in[p]) {
            const float4 *from = (const float4 *)(a.weight + (a.weight_heads ? col : 0) + 8 * (p * L + l));
            const float4 u = from[0], v = from[1];
            w[p][0] = u.x; w[p][1] = u.y; w[p][2] = u.z; w[p][3] = u.w;
            w[p][4] = v.x; w[p][5] = v.y; w[p][6] = v.z; w[p][7] = v.w;
        }
    }
    const char *x = a.x + t * a.x_stride + (col + 8 * l) * Tok<XB>::BYTES;
    const char *second = a.second + t * a.second_stride + (col + 8 * l) * Tok<SB>::BYTES;
    char *sum = GATE ? nullptr : a.sum + t * a.sum_stride + 8 * l * Tok<SB>::BYTES;
    const int width = a.out_type == LQ_TOKEN_E4M3 ? 1 : a.out_type == LQ_TOKEN_BF16 ? 2 : 4;
    char *out = a.out + t * a.out_stride + (col + 8 * l) * width;
    float *scale = a.scale + t * a.scale_stride + (col + 8 * l) / BLOCK;
    const bool with_second = GATE || a.second, with_sum = !GATE && a.sum;
    for (; t < a.tokens; t += a.step) {
        Raw<XB> xr[P];
        Raw<SB> sr[P];
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in[p]) {
                xr[p].load(x + p * (8 * L * Tok<XB>::BYTES));
                if (with_second) sr[p].load(second + p * (8 * L * Tok<SB>::BYTES));
            }
        float y[P][8], ss = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!in[p]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] = 0.0f;
                continue;
            }
            float s[8];
            xr[p].values(y[p]);
            if (with_second) sr[p].values(s);
            if (GATE) {
                gate_values(s, a.act);
                if (a.first) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[p][i] *= s[i];
                }
            } else if (with_second) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] += s[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(y[p][i], y[p][i], ss);
            if (GATE && !a.first) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] *= s[i];
            }
            if (with_sum) store_tok<SB, 8>(sum + p * (8 * L * Tok<SB>::BYTES), y[p]);
        }
        if (GATE || a.norm) {
            const float inv = 1.0f / sqrtf(row_sum<L>(ss, sums) / (float)a.length + a.eps);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] = y[p][i] * inv * w[p][i];
        }
        if (a.out_type == LQ_TOKEN_E4M3) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float most = block_most(row16_most(in[p] ? most8(y[p]) : 0u));
                const uint2 code = encode_e4m3(y[p], E4M3_MAX / most);
                if (in[p]) {
                    *(uint2 *)(out + p * 8 * L) = code;
                    if (l16 == 0) scale[p * 8 * L / BLOCK] = most / E4M3_MAX;
                }
            }
        } else if (a.out_type == LQ_TOKEN_BF16) {
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in[p]) store_tok<true, 8>(out + p * 16 * L, y[p]);
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in[p]) store_tok<false, 8>(out + p * 32 * L, y[p]);
        }
        x += a.step * a.x_stride;
        second += a.step * a.second_stride;
        if (!GATE) sum += a.step * a.sum_stride;
        out += a.step * a.out_stride;
        scale += a.step * a.scale_stride;
    }
}

// Workgroups: as many as the GPU holds at once, and tokens in turn beyond that.
constexpr uint32_t MOST_GROUPS = 256 * 8;

template <int L, int P, bool GATE>
hipError_t launch(RowArgs a, bool xb, bool sb, hipStream_t st) {
    constexpr int threads = L > 256 ? L : 256, per = threads / L;
    if (a.tokens == 0) return hipSuccess;
    a.step = std::min(a.tokens, std::max(1u, MOST_GROUPS * per / a.heads_turn));
    const dim3 grid((a.step * a.heads_turn - 1) / per + 1), block(threads);
    if (xb && sb) hipLaunchKernelGGL((rows_kernel<L, P, true, true, GATE>), grid, block, 0, st, a);
    else if (xb) hipLaunchKernelGGL((rows_kernel<L, P, true, false, GATE>), grid, block, 0, st, a);
    else if (sb) hipLaunchKernelGGL((rows_kernel<L, P, false, true, GATE>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rows_kernel<L, P, false, false, GATE>), grid, block, 0, st, a);
    return hipGetLastError();
}

// Rows longer than the 32 lanes of a head: a wave, or a workgroup, with as many pieces a lane as it takes (their
// values, weights and loads are 40 registers each).
template <bool GATE>
hipError_t launch_long(const RowArgs &a, bool xb, bool sb, hipStream_t st) {
    if (a.length <= 512) return launch<64, 1, GATE>(a, xb, sb, st);
    if (a.length <= 1024) return launch<64, 2, GATE>(a, xb, sb, st);
    if (a.length <= 2048) return launch<64, 4, GATE>(a, xb, sb, st);
    if (a.length <= 4096) return launch<256, 2, GATE>(a, xb, sb, st);
    if (a.length <= 8192) return launch<256, 4, GATE>(a, xb, sb, st);
    return launch<1024, 2, GATE>(a, xb, sb, st);    // (LQ_MAX_NORM_CHANNELS)
}

// ---- weights --------------------------------------------------------------------
//
// Bound: HBM.  A workgroup per block of 128 x 128, which stays in registers between its largest magnitude and its codes:
// 16 lanes a row of the block, 16 rows at a time.  12288 x 4096 bf16 30 us (5.0 TB/s).
struct WeightArgs {
    const char *w;
    char *out;
    float *scale;
    int64_t w_stride, out_stride;       // bytes
    int32_t n, k, blocks_k;
};

template <bool BF>
__global__ __launch_bounds__(256) void quantize_weight_kernel(WeightArgs a) {
    __shared__ uint32_t mosts[4];
    const int bn = blockIdx.x / a.blocks_k, bk = blockIdx.x - bn * a.blocks_k;
    const int r = threadIdx.x >> 4, c = bk * BLOCK + 8 * (threadIdx.x & 15);
    Raw<BF> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = bn * BLOCK + 16 * i + r;
        if (row < a.n && c < a.k) raw[i].load(a.w + row * a.w_stride + (int64_t)c * Tok<BF>::BYTES);
        else
            for (auto &p : raw[i].p) p = make_uint4(0, 0, 0, 0);
    }
    float y[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        raw[i].values(y[i]);
        m = most8(y[i], m);
    }
    m = row16_most(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((threadIdx.x & 63) == 0) mosts[threadIdx.x >> 6] = m;
    __syncthreads();
    const float most = block_most(max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3])));
    const float factor = E4M3_MAX / most;
    if (threadIdx.x == 0) a.scale[blockIdx.x] = most / E4M3_MAX;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = bn * BLOCK + 16 * i + r;
        if (row < a.n && c < a.k) *(uint2 *)(a.out + row * a.out_stride + c) = encode_e4m3(y[i], factor);
    }
}

int64_t type_size(int32_t t) { return t == LQ_TOKEN_F32 ? 4 : t == LQ_TOKEN_BF16 ? 2 : 1; }

}  // namespace

hipError_t launch_add_norm(const lq_add &n, hipStream_t st) {
    RowArgs a = {};
    a.x = (const char *)n.x;
    a.second = (const char *)n.residual;
    a.weight = n.weight;
    a.sum = (char *)n.residual_out;
    a.out = (char *)n.out;
    a.scale = n.scale;
    a.x_stride = row_bytes(n.tokens, n.x_stride, type_size(n.dtype));
    a.second_stride = n.residual ? row_bytes(n.tokens, n.residual_stride, type_size(n.residual_dtype)) : 0;
    a.sum_stride = n.residual_out ? row_bytes(n.tokens, n.residual_out_stride, type_size(n.residual_dtype)) : 0;
    a.out_stride = row_bytes(n.tokens, n.out_stride, type_size(n.out_dtype));
    a.scale_stride = row_bytes(n.tokens, n.scale_stride, 1);
    a.tokens = (uint32_t)n.tokens;
    a.heads = a.heads_turn = 1;
    a.length = n.channels;
    a.norm = n.norm == LQ_NORM_RMS;
    a.out_type = n.out_dtype;
    a.eps = n.eps;
    return launch_long<false>(a, n.dtype == LQ_TOKEN_BF16, n.residual_dtype == LQ_TOKEN_BF16, st);
}

hipError_t launch_gate_norm(const lq_gated &g, hipStream_t st) {
    RowArgs a = {};
    a.x = (const char *)g.x;
    a.second = (const char *)g.gate;
    a.weight = g.weight;
    a.out = (char *)g.out;
    a.scale = g.scale;
    a.x_stride = row_bytes(g.tokens, g.x_stride, type_size(g.dtype));
    a.second_stride = row_bytes(g.tokens, g.gate_stride, type_size(g.gate_dtype));
    a.out_stride = row_bytes(g.tokens, g.out_stride, type_size(g.out_dtype));
    a.scale_stride = row_bytes(g.tokens, g.scale_stride, 1);
    a.heads = (uint32_t)g.heads;
    // two heads of 64 share a block: a token's heads start at an even place
    a.heads_turn = g.d == 64 ? a.heads + (a.heads & 1) : a.heads;
    a.tokens = (uint32_t)g.tokens;
    a.length = g.d;
    a.norm = 1;
    a.out_type = g.out_dtype;
    a.act = g.act;
    a.first = g.gate_first;
    a.weight_heads = g.weight ? g.weight_heads : 0;
    a.eps = g.eps;
    const bool xb = g.dtype == LQ_TOKEN_BF16, gb = g.gate_dtype == LQ_TOKEN_BF16;
    switch (g.d) {
        case 64: return launch<8, 1, true>(a, xb, gb, st);
        case 128: return launch<16, 1, true>(a, xb, gb, st);
        case 256: return launch<32, 1, true>(a, xb, gb, st);
        default: return launch_long<true>(a, xb, gb, st);
    }
}

hipError_t launch_quantize_weight(const lq_weight &w, hipStream_t st) {
    WeightArgs a;
    a.w = (const char *)w.w;
    a.out = (char *)w.out;
    a.scale = w.scale;
    a.w_stride = row_bytes(w.n, w.w_stride, type_size(w.dtype));
    a.out_stride = row_bytes(w.n, w.out_stride, 1);
    a.n = w.n;
    a.k = w.k;
    a.blocks_k = (w.k + BLOCK - 1) / BLOCK;
    const dim3 grid((unsigned)((int64_t)((w.n - 1) / BLOCK + 1) * a.blocks_k));
    if (w.dtype == LQ_TOKEN_BF16) hipLaunchKernelGGL((quantize_weight_kernel<true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((quantize_weight_kernel<false>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace lq
