// Norm of queries and keys per head, and the rotation of their first channels
// by the token's position, in one pass.
//
// Bound: HBM.  A lane owns 8 channels, d/8 neighbouring lanes a head, so the
// sum of squares stays in registers (DPP, one swap for d = 256) and the other
// half of a rotated pair is in the lane itself (interleaved) or comes from a
// lane of the same head.  8192 tokens x 32 heads of 128, bf16: 31.5 us (4.3 TB/s;
// 28 at the rate of a large copy).
#include "lq_layer.hpp"
#include "lq_internal.hpp"

namespace lq {

namespace {

struct NormArgs {
    const char *in[2];          // queries, keys
    char *out[2];
    const float *weight[2];
    const float *cos, *sin;
    const int32_t *positions;
    int32_t *err;
    int64_t in_stride[2], out_stride[2];    // bytes
    int64_t rows;               // tokens * heads
    int32_t heads_q, heads, norm, rot, interleaved, n_positions;
    float eps, q_scale;
};

// Sum over the L = 8, 16 or 32 lanes of a head.
template <int L>
__device__ __forceinline__ float head_sum(float x) {
    x += dpp<DPP_XOR1>(x);
    x += dpp<DPP_XOR2>(x);
    if (L == 8) return x + dpp<DPP_HALF_MIRROR>(x);
    x += dpp<DPP_ROR4>(x);
    x += dpp<DPP_ROR8>(x);
    if (L == 32) x += __shfl_xor(x, 16);
    return x;
}

template <int DH, bool BF, bool OBF>
__global__ __launch_bounds__(256) void qk_norm_kernel(NormArgs a) {
    constexpr int L = DH / 8;
    const int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int l = threadIdx.x % L;
    const bool here = row < a.rows;             // (every lane takes part in the exchanges)
    const int64_t r = here ? row : a.rows - 1;
    const int64_t t = r / a.heads;
    const int head = (int)(r - t * a.heads);
    const int which = head >= a.heads_q;
    const int h = which ? head - a.heads_q : head;
    const char *in = a.in[which] + t * a.in_stride[which] + ((int64_t)h * DH + 8 * l) * Tok<BF>::BYTES;
    float x[8];
    unpack16<BF>(*(const uint4 *)in, x);
    if (!BF) unpack16<BF>(((const uint4 *)in)[1], x + 4);

    if (a.norm != LQ_NORM_NONE) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
        ss = head_sum<L>(ss);
        if (a.norm == LQ_NORM_RMS) ss *= 1.0f / DH;
        const float inv = 1.0f / sqrtf(ss + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv;
        const float *w = a.weight[which];
        if (w) {
            const float4 w0 = ((const float4 *)(w + 8 * l))[0], w1 = ((const float4 *)(w + 8 * l))[1];
            x[0] *= w0.x; x[1] *= w0.y; x[2] *= w0.z; x[3] *= w0.w;
            x[4] *= w1.x; x[5] *= w1.y; x[6] *= w1.z; x[7] *= w1.w;
        }
    }
    if (a.rot) {
        const int half = a.rot / 2;
        const int p = a.positions[t];
        const bool known = p >= 0 && p < a.n_positions;
        if (!known && here && l == 0 && a.err) atomicOr(a.err, LQ_DEVERR_BAD_POSITION);
        const int64_t at = (int64_t)(known ? p : 0) * half;
        if (a.interleaved) {
            if (8 * l < a.rot) {
                const float4 c = *(const float4 *)(a.cos + at + 4 * l), s = *(const float4 *)(a.sin + at + 4 * l);
                const float cc[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = x[2 * i], v = x[2 * i + 1];
                    x[2 * i] = u * cc[i] - v * sn[i];
                    x[2 * i + 1] = v * cc[i] + u * sn[i];
                }
            }
        } else {
            // rot is a multiple of 16: a lane's 8 channels lie in one half
            const bool lower = 8 * l < half, rotates = 8 * l < a.rot;
            const int j = rotates ? (lower ? 8 * l : 8 * l - half) : 0;
            const int lanes = half / 8;
            const int partner = (int)(threadIdx.x & 63) + (rotates ? (lower ? lanes : -lanes) : 0);
            float y[8], cc[8], sn[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 c = ((const float4 *)(a.cos + at + j))[i], s = ((const float4 *)(a.sin + at + j))[i];
                cc[4 * i] = c.x; cc[4 * i + 1] = c.y; cc[4 * i + 2] = c.z; cc[4 * i + 3] = c.w;
                sn[4 * i] = s.x; sn[4 * i + 1] = s.y; sn[4 * i + 2] = s.z; sn[4 * i + 3] = s.w;
            }
            if (rotates) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * cc[i] + (lower ? -y[i] : y[i]) * sn[i];
            }
        }
        if (!known && 8 * l < a.rot) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = nanf32();
        }
    }
    if (!which) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= a.q_scale;
    }
    if (here) {
        char *out = a.out[which] + t * a.out_stride[which] + ((int64_t)h * DH + 8 * l) * Tok<OBF>::BYTES;
        store_tok<OBF, 8>(out, x);
    }
}

template <int DH, bool BF, bool OBF>
hipError_t launch(const NormArgs &a, hipStream_t st) {
    constexpr int per = 256 / (DH / 8);
    if (a.rows == 0) return hipSuccess;
    hipLaunchKernelGGL((qk_norm_kernel<DH, BF, OBF>), dim3((unsigned)((a.rows + per - 1) / per)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int DH>
hipError_t launch_types(const NormArgs &a, const lq_qk &n, hipStream_t st) {
    const bool obf = n.out_dtype == LQ_TOKEN_BF16;
    if (n.dtype == LQ_TOKEN_BF16) return obf ? launch<DH, true, true>(a, st) : launch<DH, true, false>(a, st);
    return obf ? launch<DH, false, true>(a, st) : launch<DH, false, false>(a, st);
}

}  // namespace

hipError_t launch_qk_norm(const lq_qk &n, hipStream_t st) {
    NormArgs a;
    const int64_t es = n.dtype == LQ_TOKEN_BF16 ? 2 : 4, eo = n.out_dtype == LQ_TOKEN_BF16 ? 2 : 4;
    a.in[0] = (const char *)n.q;
    a.in[1] = (const char *)n.k;
    a.out[0] = (char *)n.q_out;
    a.out[1] = (char *)n.k_out;
    a.weight[0] = n.norm == LQ_NORM_RMS ? n.q_weight : nullptr;
    a.weight[1] = n.norm == LQ_NORM_RMS ? n.k_weight : nullptr;
    a.cos = n.cos;
    a.sin = n.sin;
    a.positions = n.positions;
    a.err = n.err;
    const int64_t rows_k = n.heads_k ? n.tokens : 0;
    a.in_stride[0] = row_bytes(n.tokens, n.q_stride, es);
    a.in_stride[1] = row_bytes(rows_k, n.k_stride, es);
    a.out_stride[0] = row_bytes(n.tokens, n.q_out_stride, eo);
    a.out_stride[1] = row_bytes(rows_k, n.k_out_stride, eo);
    a.heads_q = n.heads_q;
    a.heads = n.heads_q + n.heads_k;
    a.rows = n.tokens * a.heads;
    a.norm = n.norm;
    a.rot = n.rot;
    a.interleaved = n.interleaved;
    a.n_positions = n.n_positions;
    a.eps = n.eps;
    a.q_scale = n.q_scale;
    switch (n.d) {
        case 64: return launch_types<64>(a, n, st);
        case 128: return launch_types<128>(a, n, st);
        default: return launch_types<256>(a, n, st);
    }
}

}  // namespace lq
