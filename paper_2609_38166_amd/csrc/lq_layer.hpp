// Device helpers of the layer operators (convolution, query/key norm, scan):
// tokens in fp32 or bf16, packed sequences, state slots.
#pragma once

#include "leapquant.h"
#include "lq_device.hpp"

namespace lq {

// 16 bytes of token values as floats: 8 bf16 or 4 fp32.
template <bool BF> struct Tok {
    static constexpr int V = BF ? 8 : 4;
    static constexpr int BYTES = BF ? 2 : 4;
};
template <bool BF>
__device__ __forceinline__ void unpack16(const uint4 &p, float *f) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            f[i] = __uint_as_float(w[i]);
        }
    }
}

// Two floats to packed bf16 (nearest even; NaN stays NaN), lower half first.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// V consecutive floats to memory in the token type (16 or 32 bytes, aligned to 16).
template <bool BF, int V>
__device__ __forceinline__ void store_tok(void *p, const float *f) {
    if (BF) {
        if (V == 8)
            *(uint4 *)p = make_uint4(pk_bf16(f[0], f[1]), pk_bf16(f[2], f[3]), pk_bf16(f[4], f[5]), pk_bf16(f[6], f[7]));
        else
            *(uint2 *)p = make_uint2(pk_bf16(f[0], f[1]), pk_bf16(f[2], f[3]));
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) ((float4 *)p)[i / 4] = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
    }
}

// As dma16 (lq_device.hpp), one element of 2 or 4 bytes per lane: lane L writes lds_base + 4 L.
template <int BYTES>
__device__ __forceinline__ void dma_element(const void *g, uint32_t lds_base) {
    if (BYTES == 2) asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_ushort %0, off" :: "v"(g), "s"(lds_base) : "memory");
    else asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" :: "v"(g), "s"(lds_base) : "memory");
}

template <bool BF>
__device__ __forceinline__ float load_tok(const void *p, int64_t i) {
    return BF ? bf2f(((const uint16_t *)p)[i]) : ((const float *)p)[i];
}

// Tokens [begin, end) of sequence b, clamped into [0, tokens].
struct Span {
    int64_t begin, end;
};
__device__ __forceinline__ Span sequence_span(const int32_t *cu, int b, int64_t tokens) {
    const int64_t c0 = cu[b], c1 = cu[b + 1];
    Span s;
    s.begin = c0 < 0 ? 0 : c0 > tokens ? tokens : c0;
    s.end = c1 < s.begin ? s.begin : c1 > tokens ? tokens : c1;
    return s;
}

// Raises LQ_DEVERR_BAD_SEQLENS if an entry falls or leaves [0, tokens]; one
// workgroup of a launch calls this, with all its `n` threads.
__device__ __forceinline__ void check_seqlens(const int32_t *cu, int seqs, int64_t tokens, int32_t *err, int tid, int n) {
    if (!err) return;
    for (int i = tid; i < seqs; i += n)
        if (cu[i] < 0 || cu[i + 1] < cu[i] || cu[i + 1] > tokens) atomicOr(err, LQ_DEVERR_BAD_SEQLENS);
}

// The state row of a sequence: >= 0 a row, NO_SLOT none (start from zero, do
// not keep), BAD_SLOT outside the array (start from NaN, do not keep).
enum : int { NO_SLOT = -1, BAD_SLOT = -2 };
__device__ __forceinline__ int state_row(const void *state, const int32_t *slots, int b, int n_slots, int32_t *err) {
    if (!state) return NO_SLOT;
    const int s = slots ? slots[b] : b;
    if (s < 0) return NO_SLOT;
    if (s < n_slots) return s;
    if (err) atomicOr(err, LQ_DEVERR_BAD_SLOT);
    return BAD_SLOT;
}

__device__ __forceinline__ float nanf32() { return __uint_as_float(0x7FC00000u); }

// delta = softplus(x) = max(x, 0) + log1p(exp(-|x|)), or x itself.  With e the
// exponential, log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, by its series
// 2 s (1 + s^2/3 + s^4/5 + ..): eight terms leave 9^-8 / 17 = 1.4e-9, and a small e keeps
// its relative precision.
__device__ __forceinline__ float scan_delta(float x, int softplus) {
    if (!softplus) return x;
    const float e = expf(-fabsf(x)), s = e / (2.0f + e), z = s * s;
    float p = 1.0f / 15.0f;
    p = fmaf(p, z, 1.0f / 13.0f);
    p = fmaf(p, z, 1.0f / 11.0f);
    p = fmaf(p, z, 1.0f / 9.0f);
    p = fmaf(p, z, 1.0f / 7.0f);
    p = fmaf(p, z, 1.0f / 5.0f);
    p = fmaf(p, z, 1.0f / 3.0f);
    const float l = 2.0f * fmaf(s * z, p, s);
    return (x > 0.0f || x != x ? x : 0.0f) + l;     // (0 for x = -inf, a masked token: no step, no decay)
}

// alpha = exp(x).  Near 1, where a state's memory is long and the roundings of
// many steps multiply, through expm1: expf's own error there is on one side
// (a state after 1500 steps was 8.9e-6 off with it).
__device__ __forceinline__ float scan_alpha(float x) { return x > -0.35f ? 1.0f + expm1f(x) : expf(x); }

}  // namespace lq
