// Launchers shared between the C ABI layer and the kernel translation units.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "leapquant.h"

namespace lq {

struct StatePtrs {
    void *codes;
    float *scale;
    float *smooth;
    uint16_t *comp_k;
    uint16_t *comp_u;
    uint16_t *rec_k;
    uint16_t *rec_u;
    uint16_t *rec_a;
    int32_t *rec_len;
    int32_t *err;
};

struct TokenPtrs {
    const float *q;
    const float *k;
    const float *v;
    const float *alpha;
    const float *beta;
    float *o;
    const float *b;     // read vectors [tiles][d_k] (general rule only, else null)
};

hipError_t launch_decode(const lq_dims &d, const StatePtrs &s, const TokenPtrs &t, hipStream_t st);

// decode step, then the window commit of every tile whose window it filled
hipError_t launch_decode_commit(const lq_dims &d, const StatePtrs &s, const TokenPtrs &t, hipStream_t st);

// mode: 0 = quantize given fp32 states, 1 = window commit, 2 = dequantize (read only)
enum TileMode { TILE_QUANTIZE = 0, TILE_COMMIT = 1, TILE_DEQUANT = 2 };
hipError_t launch_tile(const lq_dims &d, const StatePtrs &s, int mode, const float *S_in,
                       float *S_out, const int32_t *mask, hipStream_t st);

hipError_t launch_baseline(const lq_dims &d, void *S, int state_dtype, const TokenPtrs &t,
                           hipStream_t st);

// layer operators (the structs are checked by the C ABI layer before they get here)
hipError_t launch_conv_prompt(const lq_conv &c, hipStream_t st);
hipError_t launch_conv_step(const lq_conv &c, hipStream_t st);
hipError_t launch_qk_norm(const lq_qk &n, hipStream_t st);
size_t scan_workspace_bytes(const lq_dims &d, const lq_scan &s);
hipError_t launch_scan_prompt(const lq_dims &d, const lq_scan &s, hipStream_t st);
hipError_t launch_scan_step(const lq_dims &d, const lq_scan &s, hipStream_t st);
hipError_t launch_scan_gates(const lq_dims &d, const lq_scan &s, float *alpha, float *beta, hipStream_t st);

// projection operators (checked before they get here, likewise)
hipError_t launch_add_norm(const lq_add &a, hipStream_t st);
hipError_t launch_gate_norm(const lq_gated &g, hipStream_t st);
hipError_t launch_quantize_weight(const lq_weight &w, hipStream_t st);
hipError_t launch_matmul(const lq_matmul &m, hipStream_t st);

// Bytes between the rows of a token array; of one row's, nobody has to set a stride.
inline int64_t row_bytes(int64_t tokens, int64_t stride, int64_t size) { return tokens > 1 ? stride * size : 0; }

// host checks shared by the C ABI's source files (lq_api.hip)
int32_t check_dims(const lq_dims *d);
int32_t hip_status(hipError_t e);

}  // namespace lq
