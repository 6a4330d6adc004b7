// Selective state space scan, packed prompts and single tokens:
//   S_t = alpha_t S_{t-1} + delta_t k_t v_t^T,   o_t = S_t^T q_t + skip v_t,
// delta = softplus(dt + bias), alpha = exp(delta A), the state kept as S^T.
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

// One workgroup per (sequence, value head): the state lies in registers, 8 key
// channels of the value channels r0 + 16 m per thread, and the tokens follow
// one another.  STEP: one token per request, from the dense state in place.
template <bool STEP, bool BF, bool SBF>
__global__ __launch_bounds__(NT) void scan_tokens_kernel(ScanArgs a) {
    const int tid = threadIdx.x, l16 = tid & 15, r0 = tid >> 4;
    const int b = blockIdx.x / a.heads_v, h = blockIdx.x - b * a.heads_v;
    const int slot = state_row(a.state, a.slots, b, a.n_slots, a.err);
    Span sp{b, b + 1};
    if (!STEP) {
        if (blockIdx.x == 0) check_seqlens(a.cu, a.batch, a.tokens, a.err, tid, NT);
        sp = sequence_span(a.cu, b, a.tokens);
    }
    float s[8][8];
    char *St = a.state + ((int64_t)slot * a.heads_v + h) * D * D * (SBF ? 2 : 4);
    const bool from = slot >= 0 && (STEP || a.carry);
    const float fill = slot == BAD_SLOT ? nanf32() : 0.0f;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
        if (from) {
            load8<SBF>(St + ((r0 + 16 * m) * D + 8 * l16) * (SBF ? 2 : 4), s[m]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[m][j] = fill;
        }
    }
    const float A = a.A[h], bias = a.bias ? a.bias[h] : 0.0f, skip = a.skip ? a.skip[h] : 0.0f;
    const int64_t kc = ((int64_t)(h / a.group) * D + 8 * l16) * Tok<BF>::BYTES;
    for (int64_t t = sp.begin; t < sp.end; ++t) {
        float k[8], q[8];
        load8<BF>(a.k + t * a.k_stride + kc, k);
        load8<BF>(a.q + t * a.q_stride + kc, q);
        const float delta = scan_delta(load_tok<BF>(a.dt + t * a.dt_stride, h) + bias, a.softplus);
        const float alpha = scan_alpha(delta * A);
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] *= delta;
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            const int row = r0 + 16 * m;
            const float v = load_tok<BF>(a.v + t * a.v_stride, (int64_t)h * D + row);
            float y = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[m][j] = fmaf(k[j], v, alpha * s[m][j]);
            if (SBF) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t w = pk_bf16(s[m][j], s[m][j + 1]);
                    s[m][j] = __uint_as_float(w << 16);
                    s[m][j + 1] = __uint_as_float(w & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y = fmaf(s[m][j], q[j], y);
            y = row16_sum(y) + (a.skip ? skip * v : 0.0f);
            if (l16 == 0) {
                if (BF) ((uint16_t *)(a.o + t * a.o_stride))[h * D + row] = (uint16_t)pk_bf16(y, y);
                else ((float *)(a.o + t * a.o_stride))[h * D + row] = y;
            }
        }
    }
    if (slot >= 0) {
#pragma unroll
        for (int m = 0; m < 8; ++m) store_tok<SBF, 8>(St + ((r0 + 16 * m) * D + 8 * l16) * (SBF ? 2 : 4), s[m]);
    }
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
    a.q_stride = s.q_stride * es;
    a.k_stride = s.k_stride * es;
    a.v_stride = s.v_stride * es;
    a.dt_stride = s.dt_stride * es;
    a.o_stride = s.o_stride * es;
    a.batch = d.batch;
    a.heads_v = d.heads_v;
    a.group = d.heads_v / d.heads_k;
    a.n_slots = s.n_slots;
    a.softplus = s.softplus;
    a.carry = s.carry;
    return a;
}

}  // namespace

size_t scan_workspace_bytes(const lq_dims &, const lq_scan &) { return 0; }

hipError_t launch_scan_prompt(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    const ScanArgs a = scan_args(d, s);
    const dim3 grid(d.batch * d.heads_v);
    if (s.dtype == LQ_TOKEN_BF16) hipLaunchKernelGGL((scan_tokens_kernel<false, true, false>), grid, dim3(NT), 0, st, a);
    else hipLaunchKernelGGL((scan_tokens_kernel<false, false, false>), grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_scan_step(const lq_dims &d, const lq_scan &s, hipStream_t st) {
    const ScanArgs a = scan_args(d, s);
    const dim3 grid(d.batch * d.heads_v);
    const bool sbf = s.state_dtype == LQ_STATE_BF16;
    if (s.dtype == LQ_TOKEN_BF16) {
        if (sbf) hipLaunchKernelGGL((scan_tokens_kernel<true, true, true>), grid, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL((scan_tokens_kernel<true, true, false>), grid, dim3(NT), 0, st, a);
    } else {
        if (sbf) hipLaunchKernelGGL((scan_tokens_kernel<true, false, true>), grid, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL((scan_tokens_kernel<true, false, false>), grid, dim3(NT), 0, st, a);
    }
    return hipGetLastError();
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
