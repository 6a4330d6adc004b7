// C ABI of the layer operators: host-side validation and launches, under the
// rules of lq_api.hip (arguments are checked completely before anything is
// enqueued; nothing is allocated, nothing waits).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "leapquant.h"
#include "lq_checks.hpp"
#include "lq_internal.hpp"

namespace {

using namespace lq;

int32_t check_state(const void *state, int32_t n_slots, const int32_t *slots, int32_t seqs, bool needed) {
    int32_t e;
    if ((e = check(state, 16, needed)) != LQ_OK) return e;
    if ((e = check(slots, 4, false)) != LQ_OK) return e;
    if (state && (n_slots <= 0 || (!slots && n_slots < seqs))) return LQ_EINVAL;
    return LQ_OK;
}

int32_t check_conv(const lq_conv *c, bool step) {
    if (!c) return LQ_EINVAL;
    int32_t e;
    if (c->seqs <= 0 || c->channels <= 0 || !token_type(c->dtype) || !token_type(c->out_dtype) || !flag(c->silu) ||
        !flag(c->carry))
        return LQ_EINVAL;
    if ((e = check_tokens(c->tokens)) != LQ_OK) return e;
    if (step && c->tokens != c->seqs) return LQ_EINVAL;
    if (c->width < 2 || c->width > LQ_MAX_CONV_WIDTH) return LQ_EUNSUPPORTED;
    const int32_t per = c->dtype == LQ_TOKEN_BF16 ? 8 : 4;
    if (c->channels % per) return LQ_EUNSUPPORTED;
    // workgroups: at least 32 tokens of 64 lanes' channels (the step: a request), or 4 states
    const int64_t blocks = ((int64_t)c->channels / per + 63) / 64 * ((c->tokens + 31) / 32 + c->seqs);
    if (blocks > MAX_BLOCKS) return LQ_EUNSUPPORTED;
    if ((e = check(c->weight, 16)) != LQ_OK) return e;
    if ((e = check(c->bias, 4, false)) != LQ_OK) return e;
    if ((e = check_rows(c->x, c->tokens, c->channels, c->x_stride, token_size(c->dtype), 16)) != LQ_OK) return e;
    if ((e = check_rows(c->out, c->tokens, c->channels, c->out_stride, token_size(c->out_dtype), 16)) != LQ_OK) return e;
    if (!step && (e = check(c->cu_seqlens, 4)) != LQ_OK) return e;
    if ((e = check_state(c->state, c->n_slots, c->slots, c->seqs, step || c->carry)) != LQ_OK) return e;
    return check(c->err, 4, false);
}

// what: 0 prompt, 1 step, 2 gates
int32_t check_scan(const lq_dims *d, const lq_scan *s, int what) {
    int32_t e = lq::check_dims(d);
    if (e != LQ_OK) return e;
    if (!s) return LQ_EINVAL;
    if (!token_type(s->dtype) || !flag(s->softplus)) return LQ_EINVAL;
    if ((e = check_tokens(s->tokens)) != LQ_OK) return e;
    if (d->gate != LQ_GATE_SCALAR || d->rule != LQ_RULE_ADD) return LQ_EUNSUPPORTED;
    const int64_t es = token_size(s->dtype), T = s->tokens;
    if ((e = check(s->A, 4)) != LQ_OK) return e;
    if ((e = check(s->dt_bias, 4, false)) != LQ_OK) return e;
    if ((e = check_rows(s->dt, T, d->heads_v, s->dt_stride, es, (uintptr_t)es)) != LQ_OK) return e;
    if (what == 2) return T * d->heads_v > 256 * MAX_BLOCKS ? LQ_EUNSUPPORTED : LQ_OK;
    if ((int64_t)d->batch * d->heads_v > MAX_BLOCKS / 8) return LQ_EUNSUPPORTED;      // (up to eight workgroups a tile)
    if (s->state_dtype != LQ_STATE_F32 && s->state_dtype != LQ_STATE_BF16) return LQ_EINVAL;
    if (!flag(s->carry) || s->max_len < 0) return LQ_EINVAL;
    if (what == 1 && T != d->batch) return LQ_EINVAL;
    if (what == 0 && s->state_dtype != LQ_STATE_F32) return LQ_EUNSUPPORTED;
    const int64_t rk = (int64_t)d->heads_k * d->d_k, rv = (int64_t)d->heads_v * d->d_v;
    if ((e = check_rows(s->q, T, rk, s->q_stride, es, 16)) != LQ_OK) return e;
    if ((e = check_rows(s->k, T, rk, s->k_stride, es, 16)) != LQ_OK) return e;
    if ((e = check_rows(s->v, T, rv, s->v_stride, es, 16)) != LQ_OK) return e;
    if ((e = check_rows(s->o, T, rv, s->o_stride, es, 16)) != LQ_OK) return e;
    if ((e = check(s->skip, 4, false)) != LQ_OK) return e;
    if (what == 0 && (e = check(s->cu_seqlens, 4)) != LQ_OK) return e;
    if ((e = check_state(s->state, s->n_slots, s->slots, d->batch, what == 1 || s->carry)) != LQ_OK) return e;
    return check(s->err, 4, false);
}

}  // namespace

extern "C" {

int32_t leapquant_conv_prompt(const lq_conv *c, void *stream) {
    const int32_t e = check_conv(c, false);
    if (e != LQ_OK) return e;
    return hip_status(lq::launch_conv_prompt(*c, (hipStream_t)stream));
}

int32_t leapquant_conv_step(const lq_conv *c, void *stream) {
    const int32_t e = check_conv(c, true);
    if (e != LQ_OK) return e;
    return hip_status(lq::launch_conv_step(*c, (hipStream_t)stream));
}

int32_t leapquant_qk_norm(const lq_qk *n, void *stream) {
    if (!n) return LQ_EINVAL;
    int32_t e;
    if (n->heads_q <= 0 || n->heads_k < 0 || n->rot < 0 || !flag(n->interleaved) || !token_type(n->dtype) ||
        !token_type(n->out_dtype))
        return LQ_EINVAL;
    if (n->norm != LQ_NORM_NONE && n->norm != LQ_NORM_L2 && n->norm != LQ_NORM_RMS) return LQ_EINVAL;
    if (n->norm != LQ_NORM_RMS && (n->q_weight || n->k_weight)) return LQ_EINVAL;
    if (!(n->eps >= 0.0f) || !(n->eps <= 3.4e38f)) return LQ_EINVAL;
    if ((e = check_tokens(n->tokens)) != LQ_OK) return e;
    if (n->d != 64 && n->d != 128 && n->d != 256) return LQ_EUNSUPPORTED;
    if (n->rot % 16 || n->rot > n->d) return LQ_EUNSUPPORTED;
    if ((int64_t)n->heads_q + n->heads_k > (1 << 20)) return LQ_EUNSUPPORTED;
    if (n->tokens * ((int64_t)n->heads_q + n->heads_k) / (2048 / n->d) >= MAX_BLOCKS) return LQ_EUNSUPPORTED;
    const int64_t es = token_size(n->dtype), eo = token_size(n->out_dtype);
    const int64_t rq = (int64_t)n->heads_q * n->d, rk = (int64_t)n->heads_k * n->d;
    if ((e = check_rows(n->q, n->tokens, rq, n->q_stride, es, 16)) != LQ_OK) return e;
    if ((e = check_rows(n->q_out, n->tokens, rq, n->q_out_stride, eo, 16)) != LQ_OK) return e;
    if (n->heads_k) {
        if ((e = check_rows(n->k, n->tokens, rk, n->k_stride, es, 16)) != LQ_OK) return e;
        if ((e = check_rows(n->k_out, n->tokens, rk, n->k_out_stride, eo, 16)) != LQ_OK) return e;
    }
    if ((e = check(n->q_weight, 16, false)) != LQ_OK) return e;
    if ((e = check(n->k_weight, 16, false)) != LQ_OK) return e;
    if (n->rot) {
        if (n->n_positions <= 0) return LQ_EINVAL;
        if ((e = check(n->cos, 16)) != LQ_OK) return e;
        if ((e = check(n->sin, 16)) != LQ_OK) return e;
        if (n->tokens && (e = check(n->positions, 4)) != LQ_OK) return e;
    }
    if ((e = check(n->err, 4, false)) != LQ_OK) return e;
    return hip_status(lq::launch_qk_norm(*n, (hipStream_t)stream));
}

int32_t leapquant_scan_workspace_bytes(const lq_dims *d, const lq_scan *s, size_t *bytes_out) {
    int32_t e = lq::check_dims(d);
    if (e != LQ_OK) return e;
    if (!s || !bytes_out || !token_type(s->dtype) || s->max_len < 0) return LQ_EINVAL;
    if ((e = check_tokens(s->tokens)) != LQ_OK) return e;
    *bytes_out = lq::scan_workspace_bytes(*d, *s);
    return LQ_OK;
}

int32_t leapquant_scan_prompt(const lq_dims *d, const lq_scan *s, void *stream) {
    int32_t e = check_scan(d, s, 0);
    if (e != LQ_OK) return e;
    lq_scan one = *s;                           // (this call alone, not all that max_len = 0 stands for)
    if (one.max_len == 0) one.max_len = (int32_t)one.tokens;
    if (lq::scan_workspace_bytes(*d, one)) {
        const size_t need = lq::scan_workspace_bytes(*d, *s);
        if ((e = check(s->workspace, 16)) != LQ_OK) return e;
        if (s->workspace_bytes < need) return LQ_EINVAL;
    }
    return hip_status(lq::launch_scan_prompt(*d, *s, (hipStream_t)stream));
}

int32_t leapquant_scan_step(const lq_dims *d, const lq_scan *s, void *stream) {
    const int32_t e = check_scan(d, s, 1);
    if (e != LQ_OK) return e;
    return hip_status(lq::launch_scan_step(*d, *s, (hipStream_t)stream));
}

int32_t leapquant_scan_gates(const lq_dims *d, const lq_scan *s, float *alpha, float *beta, void *stream) {
    int32_t e = check_scan(d, s, 2);
    if (e != LQ_OK) return e;
    if (s->tokens == 0) return LQ_OK;
    if ((e = check(alpha, 4)) != LQ_OK) return e;
    if ((e = check(beta, 4)) != LQ_OK) return e;
    return hip_status(lq::launch_scan_gates(*d, *s, alpha, beta, (hipStream_t)stream));
}

}  // extern "C"
