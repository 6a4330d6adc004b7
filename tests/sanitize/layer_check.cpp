// Memory and undefined-behaviour check of the layer operators' host code (test infrastructure).
//
// tests/test_layer_sanitizers.py compiles the host layer (lq_api.hip and lq_layer_api.hip, host pass only) with
// AddressSanitizer and UndefinedBehaviorSanitizer and links it with this driver, whose launchers only record that they were
// reached: valid calls must reach them, and every rejection must not.  Pointers are plain addresses, never dereferenced.
#include <cstdio>
#include <cstdint>

#include "leapquant.h"
#include "lq_internal.hpp"

namespace {
int launches = 0;
hipError_t next_status = hipSuccess;
size_t need = 0;
}  // namespace

namespace lq {
hipError_t launch_decode(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_commit(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_tile(const lq_dims &, const StatePtrs &, int, const float *, float *, const int32_t *, hipStream_t) { return hipSuccess; }
hipError_t launch_baseline(const lq_dims &, void *, int, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_conv_prompt(const lq_conv &, hipStream_t) { ++launches; return next_status; }
hipError_t launch_conv_step(const lq_conv &, hipStream_t) { ++launches; return next_status; }
hipError_t launch_qk_norm(const lq_qk &, hipStream_t) { ++launches; return next_status; }
size_t scan_workspace_bytes(const lq_dims &, const lq_scan &) { return need; }
hipError_t launch_scan_prompt(const lq_dims &, const lq_scan &, hipStream_t) { ++launches; return next_status; }
hipError_t launch_scan_step(const lq_dims &, const lq_scan &, hipStream_t) { ++launches; return next_status; }
hipError_t launch_scan_gates(const lq_dims &, const lq_scan &, float *, float *, hipStream_t) { ++launches; return next_status; }
}  // namespace lq

namespace {

int failures = 0;
void expect(bool ok, const char *what, int line) {
    if (!ok) {
        std::fprintf(stderr, "line %d: %s\n", line, what);
        ++failures;
    }
}
#define EXPECT(c) expect((c), #c, __LINE__)

template <typename T>
T *P(uintptr_t a = 0x10000) { return reinterpret_cast<T *>(a); }

lq_conv conv() {
    lq_conv c = {};
    c.seqs = c.n_slots = 3;
    c.channels = 256;
    c.width = 4;
    c.dtype = LQ_TOKEN_BF16;
    c.silu = c.carry = 1;
    c.tokens = 3;
    c.x_stride = c.out_stride = 256;
    c.x = P<void>();
    c.weight = P<float>();
    c.out = P<void>();
    c.state = P<void>();
    c.cu_seqlens = P<int32_t>();
    return c;
}
lq_qk qk() {
    lq_qk n = {};
    n.tokens = 7;
    n.heads_q = 2;
    n.heads_k = 1;
    n.d = 64;
    n.rot = 32;
    n.norm = LQ_NORM_L2;
    n.q_stride = n.q_out_stride = 128;
    n.k_stride = n.k_out_stride = 64;
    n.q = n.k = P<void>();
    n.q_out = n.k_out = P<void>();
    n.cos = n.sin = P<float>();
    n.positions = P<int32_t>();
    n.n_positions = 4;
    n.q_scale = 1.0f;
    return n;
}
lq_dims dims() {
    lq_dims d = {};
    d.batch = 2;
    d.heads_v = 4;
    d.heads_k = 2;
    d.d_k = d.d_v = 128;
    d.window = 1;
    d.rule = LQ_RULE_ADD;
    return d;
}
lq_scan scan() {
    lq_scan s = {};
    s.tokens = s.n_slots = 2;
    s.dtype = LQ_TOKEN_F32;
    s.q_stride = s.k_stride = 256;
    s.v_stride = s.o_stride = 512;
    s.dt_stride = 4;
    s.q = s.k = s.v = s.dt = P<void>();
    s.A = P<float>();
    s.o = s.state = P<void>();
    s.cu_seqlens = P<int32_t>();
    return s;
}

void valid_calls() {
    const int before = launches;
    lq_conv c = conv();
    lq_qk n = qk();
    lq_dims d = dims();
    lq_scan s = scan();
    EXPECT(leapquant_conv_prompt(&c, nullptr) == LQ_OK);
    EXPECT(leapquant_conv_step(&c, nullptr) == LQ_OK);
    EXPECT(leapquant_qk_norm(&n, nullptr) == LQ_OK);
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_OK);
    EXPECT(leapquant_scan_step(&d, &s, nullptr) == LQ_OK);
    EXPECT(leapquant_scan_gates(&d, &s, P<float>(), P<float>(), nullptr) == LQ_OK);
    // no tokens, no state: the arrays may be absent
    c.tokens = 0;
    c.x = nullptr;
    c.out = nullptr;
    c.state = nullptr;
    c.carry = 0;
    EXPECT(leapquant_conv_prompt(&c, nullptr) == LQ_OK);
    n.tokens = 0;
    n.q = n.k = nullptr;
    n.q_out = n.k_out = nullptr;
    n.positions = nullptr;
    EXPECT(leapquant_qk_norm(&n, nullptr) == LQ_OK);
    s.tokens = 0;
    s.q = s.k = s.v = s.dt = nullptr;
    s.o = s.state = nullptr;
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_OK);
    EXPECT(leapquant_scan_gates(&d, &s, nullptr, nullptr, nullptr) == LQ_OK);     // (nothing to launch)
    EXPECT(launches == before + 9);
    s = scan();
    next_status = hipErrorInvalidValue;
    EXPECT(leapquant_scan_step(&d, &s, nullptr) == LQ_EHIP);
    next_status = hipSuccess;
}

void rejections() {
    const int before = launches;
    lq_dims d = dims();
    for (int i = 0; i < 18; ++i) {
        lq_conv c = conv();
        switch (i) {
            case 0: c.seqs = -1; break;
            case 1: c.channels = INT32_MAX; break;
            case 2: c.width = INT32_MIN; break;
            case 3: c.tokens = INT64_MAX; break;
            case 4: c.x_stride = INT64_MAX; break;
            case 5: c.x_stride = INT64_MIN; break;
            case 6: c.n_slots = INT32_MIN; break;
            case 7: c.x = P<void>(0x10001); break;
            case 8: c.out_dtype = 9; break;
            case 9: c.seqs = INT32_MAX; c.tokens = INT32_MAX; break;
            case 10: c.weight = nullptr; break;
            case 11: c.slots = P<int32_t>(0x10002); break;
            case 12: c.err = P<int32_t>(0x10003); break;
            case 13: c.channels = 0; break;
            case 14: c.carry = 2; break;
            case 15: c.silu = -1; break;
            case 16: c.out_stride = 8; break;
            default: c.state = P<void>(0x10008); break;
        }
        EXPECT(leapquant_conv_prompt(&c, nullptr) < 0);
        EXPECT(leapquant_conv_step(&c, nullptr) < 0);
    }
    for (int i = 0; i < 12; ++i) {
        lq_qk n = qk();
        switch (i) {
            case 0: n.tokens = INT64_MAX; break;
            case 1: n.heads_q = INT32_MAX; n.heads_k = INT32_MAX; break;
            case 2: n.heads_q = 0; break;
            case 3: n.d = INT32_MIN; break;
            case 4: n.rot = INT32_MIN; break;
            case 5: n.rot = INT32_MAX; break;
            case 6: n.q_stride = INT64_MAX; break;
            case 7: n.eps = -0.5f; break;
            case 8: n.n_positions = INT32_MIN; break;
            case 9: n.tokens = INT32_MAX; n.heads_q = 1 << 19; n.q_stride = n.q_out_stride = 1LL << 30; break;
            case 10: n.k_weight = P<float>(); break;
            default: n.norm = INT32_MAX; break;
        }
        EXPECT(leapquant_qk_norm(&n, nullptr) < 0);
    }
    for (int i = 0; i < 14; ++i) {
        lq_scan s = scan();
        lq_dims e = dims();
        switch (i) {
            case 0: s.tokens = INT64_MAX; break;
            case 1: s.tokens = -1; break;
            case 2: s.dt_stride = INT64_MAX; break;
            case 3: s.max_len = INT32_MIN; break;
            case 4: s.n_slots = INT32_MIN; break;
            case 5: e.batch = 1 << 26; e.heads_k = e.heads_v; s.tokens = e.batch; s.n_slots = e.batch; break;
            case 6: s.state_dtype = INT32_MAX; break;
            case 7: s.dt = P<void>(0x10002); break;
            case 8: s.A = nullptr; break;
            case 9: e.gate = LQ_GATE_DIAG; break;
            case 10: e.rule = LQ_RULE_DELTA; break;
            case 11: s.softplus = 7; break;
            case 12: s.o = P<void>(0x10004); break;
            default: s.carry = 5; break;
        }
        EXPECT(leapquant_scan_prompt(&e, &s, nullptr) < 0);
        EXPECT(leapquant_scan_step(&e, &s, nullptr) < 0);
    }
    lq_scan s = scan();
    need = 4096;
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_EINVAL);
    s.workspace = P<void>(0x10008);
    s.workspace_bytes = need;
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_EALIGN);
    s.workspace = P<void>();
    s.workspace_bytes = need - 1;
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_EINVAL);
    EXPECT(launches == before);
    s.workspace_bytes = need;
    EXPECT(leapquant_scan_prompt(&d, &s, nullptr) == LQ_OK);
    size_t bytes = 0;
    EXPECT(leapquant_scan_workspace_bytes(&d, &s, &bytes) == LQ_OK && bytes == need);
    EXPECT(leapquant_scan_workspace_bytes(&d, &s, nullptr) == LQ_EINVAL);
    need = 0;
}

}  // namespace

int main() {
    valid_calls();
    rejections();
    if (failures) {
        std::fprintf(stderr, "%d failures\n", failures);
        return 1;
    }
    std::printf("layer sanitizer check ok (%d launches)\n", launches);
    return 0;
}
