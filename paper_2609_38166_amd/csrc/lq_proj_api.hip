// C ABI of the projection operators: host-side validation and launches, under the rules of lq_api.hip (arguments are checked
// completely before anything is enqueued; nothing is allocated, nothing waits).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "leapquant.h"
#include "lq_checks.hpp"
#include "lq_internal.hpp"

namespace {

using namespace lq;

int64_t out_size(int32_t t) { return t == LQ_TOKEN_E4M3 ? 1 : token_size(t); }
bool out_type(int32_t t) { return token_type(t) || t == LQ_TOKEN_E4M3; }

bool epsilon(float x) { return x >= 0.0f && x <= 3.4e38f; }     // (not NaN)

// Scales of E4M3 rows: fp32 rows of `blocks`, read and written one at a time.
int32_t check_scales(const float *p, int64_t tokens, int64_t channels, int64_t stride) {
    return check_rows(p, tokens, (channels + LQ_SCALE_BLOCK - 1) / LQ_SCALE_BLOCK, stride, 4, 4);
}

}  // namespace

extern "C" {

int32_t leapquant_add_norm(const lq_add *a, void *stream) {
    if (!a) return LQ_EINVAL;
    int32_t e;
    if (a->channels <= 0 || !token_type(a->dtype) || !token_type(a->residual_dtype) || !out_type(a->out_dtype)) return LQ_EINVAL;
    if (a->norm != LQ_NORM_NONE && a->norm != LQ_NORM_RMS) return LQ_EINVAL;
    if (a->norm != LQ_NORM_RMS && a->weight) return LQ_EINVAL;
    if (!epsilon(a->eps)) return LQ_EINVAL;
    if ((e = check_tokens(a->tokens)) != LQ_OK) return e;
    if (a->channels % 8 || a->channels > LQ_MAX_NORM_CHANNELS) return LQ_EUNSUPPORTED;
    const int64_t T = a->tokens, c = a->channels, es = token_size(a->dtype), er = token_size(a->residual_dtype);
    if ((e = check_rows(a->x, T, c, a->x_stride, es, 16)) != LQ_OK) return e;
    if (a->residual && (e = check_rows(a->residual, T, c, a->residual_stride, er, 16)) != LQ_OK) return e;
    if (a->residual_out && (e = check_rows(a->residual_out, T, c, a->residual_out_stride, er, 16)) != LQ_OK) return e;
    if ((e = check_rows(a->out, T, c, a->out_stride, out_size(a->out_dtype), 16)) != LQ_OK) return e;
    if ((e = check(a->weight, 16, false)) != LQ_OK) return e;
    if (a->out_dtype == LQ_TOKEN_E4M3 && (e = check_scales(a->scale, T, c, a->scale_stride)) != LQ_OK) return e;
    return hip_status(launch_add_norm(*a, (hipStream_t)stream));
}

int32_t leapquant_gate_norm(const lq_gated *g, void *stream) {
    if (!g) return LQ_EINVAL;
    int32_t e;
    if (g->heads <= 0 || g->d <= 0 || !token_type(g->dtype) || !token_type(g->gate_dtype) || !out_type(g->out_dtype)) return LQ_EINVAL;
    if (g->act != LQ_ACT_SILU && g->act != LQ_ACT_SIGMOID) return LQ_EINVAL;
    if (!flag(g->gate_first) || !flag(g->weight_heads) || !epsilon(g->eps)) return LQ_EINVAL;
    if ((e = check_tokens(g->tokens)) != LQ_OK) return e;
    if ((g->d != 64 && g->d % 128) || g->d > LQ_MAX_NORM_CHANNELS) return LQ_EUNSUPPORTED;
    if (g->heads > 1 << 20) return LQ_EUNSUPPORTED;      // (a workgroup each, at the most)
    const int64_t T = g->tokens, c = (int64_t)g->heads * g->d;
    if ((e = check_rows(g->x, T, c, g->x_stride, token_size(g->dtype), 16)) != LQ_OK) return e;
    if ((e = check_rows(g->gate, T, c, g->gate_stride, token_size(g->gate_dtype), 16)) != LQ_OK) return e;
    if ((e = check_rows(g->out, T, c, g->out_stride, out_size(g->out_dtype), 16)) != LQ_OK) return e;
    if ((e = check(g->weight, 16, false)) != LQ_OK) return e;
    if (g->out_dtype == LQ_TOKEN_E4M3 && (e = check_scales(g->scale, T, c, g->scale_stride)) != LQ_OK) return e;
    return hip_status(launch_gate_norm(*g, (hipStream_t)stream));
}

int32_t leapquant_quantize_weight(const lq_weight *w, void *stream) {
    if (!w || w->n <= 0 || w->k <= 0 || !token_type(w->dtype)) return LQ_EINVAL;
    if (w->k % 16) return LQ_EUNSUPPORTED;
    const int64_t blocks_n = ((int64_t)w->n + LQ_SCALE_BLOCK - 1) / LQ_SCALE_BLOCK;
    const int64_t blocks_k = ((int64_t)w->k + LQ_SCALE_BLOCK - 1) / LQ_SCALE_BLOCK;
    if (blocks_n * blocks_k > MAX_BLOCKS) return LQ_EUNSUPPORTED;
    int32_t e;
    if ((e = check_rows(w->w, w->n, w->k, w->w_stride, token_size(w->dtype), 16)) != LQ_OK) return e;
    if ((e = check_rows(w->out, w->n, w->k, w->out_stride, 1, 16)) != LQ_OK) return e;
    if ((e = check(w->scale, 4)) != LQ_OK) return e;
    return hip_status(launch_quantize_weight(*w, (hipStream_t)stream));
}

int32_t leapquant_matmul(const lq_matmul *m, void *stream) {
    if (!m || m->n <= 0 || m->k <= 0 || !token_type(m->out_dtype)) return LQ_EINVAL;
    int32_t e;
    if ((e = check_tokens(m->tokens)) != LQ_OK) return e;
    if (m->k % 16) return LQ_EUNSUPPORTED;
    // (a launch's work-items are counted in 32 bits, 512 of them for 16 channels of few tokens; of many tokens the tiles, of 64 x 64
    // outputs at the least, and the places that they are dealt to are 32-bit numbers)
    if (m->n > 1 << 26 || m->tokens > 1 << 28 || m->tokens > (1LL << 36) / m->n) return LQ_EUNSUPPORTED;
    // a tile's rows are addressed by 32 bits from its first one
    const int64_t T = m->tokens, apart = 1 << 23, scales_apart = 1 << 20;
    if (m->k > apart || (T > 1 && (m->x_stride > apart || m->x_scale_stride > scales_apart))) return LQ_EUNSUPPORTED;
    if (m->n > 1 && m->w_stride > apart) return LQ_EUNSUPPORTED;
    if (((int64_t)m->n + 127) / 128 * (((int64_t)m->k + 127) / 128) > 1 << 29) return LQ_EUNSUPPORTED;
    if ((e = check_rows(m->x, T, m->k, m->x_stride, 1, 16)) != LQ_OK) return e;
    if ((e = check_scales(m->x_scale, T, m->k, m->x_scale_stride)) != LQ_OK) return e;
    if ((e = check_rows(m->w, m->n, m->k, m->w_stride, 1, 16)) != LQ_OK) return e;
    if ((e = check(m->w_scale, 4)) != LQ_OK) return e;
    if ((e = check(m->bias, 4, false)) != LQ_OK) return e;
    if ((e = check_rows(m->out, T, m->n, m->out_stride, token_size(m->out_dtype), 16)) != LQ_OK) return e;
    return hip_status(launch_matmul(*m, (hipStream_t)stream));
}

}  // extern "C"
