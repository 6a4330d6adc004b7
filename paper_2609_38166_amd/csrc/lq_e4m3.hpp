// Device helpers of the projection operators: blocks of 128 values in E4M3 with a scale.
#pragma once

#include "lq_layer.hpp"

namespace lq {

constexpr int BLOCK = LQ_SCALE_BLOCK;
constexpr float E4M3_MAX = 448.0f;
// A block's largest magnitude counts as at least 2^-100, so that 448 / most and the scale stay normal numbers.
constexpr uint32_t LEAST_BITS = 27u << 23;

// Magnitudes are compared as bits: their order is that of the values, with infinity and then NaN above all of them.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t most8(const float *y, uint32_t m = 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(y[i]));
    return m;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_bits(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}
// Largest over the 16 lanes of a DPP row (8 channels a lane: a block).
__device__ __forceinline__ uint32_t row16_most(uint32_t x) {
    x = max(x, dpp_bits<DPP_XOR1>(x));
    x = max(x, dpp_bits<DPP_XOR2>(x));
    x = max(x, dpp_bits<DPP_ROR4>(x));
    return max(x, dpp_bits<DPP_ROR8>(x));
}
__device__ __forceinline__ float block_most(uint32_t bits) { return __uint_as_float(max(bits, LEAST_BITS)); }

// 8 values times 448 / most, to the nearest code.  (|y| * factor may be 448 (1 + 2^-23), which still rounds to 448.)
__device__ __forceinline__ uint2 encode_e4m3(const float *y, float factor) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] * factor, y[4 * i + 1] * factor, 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] * factor, y[4 * i + 3] * factor, lo, true);
    }
    return make_uint2(w[0], w[1]);
}

}  // namespace lq
