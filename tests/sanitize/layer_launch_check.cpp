// Undefined-behaviour check of the layer operators' launchers (test infrastructure): the arguments of calls with at most one
// token, whose strides nobody has to set, up to the launch itself, which fails for want of a GPU.
#include <cstdint>
#include <cstdio>

#include "leapquant.h"
#include "lq_internal.hpp"

namespace lq {
hipError_t launch_decode(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_commit(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_tile(const lq_dims &, const StatePtrs &, int, const float *, float *, const int32_t *, hipStream_t) { return hipSuccess; }
hipError_t launch_baseline(const lq_dims &, void *, int, const TokenPtrs &, hipStream_t) { return hipSuccess; }
}  // namespace lq

int main() {
    int n = 0;
    if (hipGetDeviceCount(&n) == hipSuccess && n > 0) {
        std::printf("a GPU is visible: nothing is launched\n");
        return 1;
    }
    int calls = 0, bad = 0;
    auto expect = [&](int32_t status) {
        ++calls;
        bad += status != LQ_EHIP;
    };
    void *const P = (void *)0x10000;
    for (int32_t type : {LQ_TOKEN_F32, LQ_TOKEN_BF16})
        for (int64_t stride : {INT64_MAX, INT64_MIN, (int64_t)0}) {
            lq_conv c = {};
            c.seqs = c.n_slots = 1;
            c.tokens = 1;
            c.channels = 64;
            c.width = 4;
            c.dtype = c.out_dtype = type;
            c.x_stride = c.out_stride = stride;
            c.x = c.out = c.state = P;
            c.weight = (const float *)P;
            c.cu_seqlens = (const int32_t *)P;
            expect(leapquant_conv_prompt(&c, nullptr));
            expect(leapquant_conv_step(&c, nullptr));
            lq_qk q = {};
            q.tokens = q.heads_q = q.heads_k = 1;
            q.d = 128;
            q.dtype = q.out_dtype = type;
            q.q_stride = q.k_stride = q.q_out_stride = q.k_out_stride = stride;
            q.q = q.k = q.q_out = q.k_out = P;
            expect(leapquant_qk_norm(&q, nullptr));
            q.heads_k = 0;                      // (nor, of several, the strides of keys that are not there)
            q.k = q.k_out = nullptr;
            expect(leapquant_qk_norm(&q, nullptr));
            lq_dims d = {};
            d.batch = d.heads_v = d.heads_k = d.window = 1;
            d.d_k = d.d_v = 128;
            d.rule = LQ_RULE_ADD;
            lq_scan s = {};
            s.tokens = s.n_slots = 1;
            s.dtype = type;
            s.q_stride = s.k_stride = s.v_stride = s.dt_stride = s.o_stride = stride;
            s.q = s.k = s.v = s.dt = s.o = s.state = P;
            s.A = (const float *)P;
            s.cu_seqlens = (const int32_t *)P;
            expect(leapquant_scan_prompt(&d, &s, nullptr));
            expect(leapquant_scan_step(&d, &s, nullptr));
            expect(leapquant_scan_gates(&d, &s, (float *)P, (float *)P, nullptr));
            q.tokens = 2;
            q.q_stride = q.q_out_stride = 128;
            expect(leapquant_qk_norm(&q, nullptr));
        }
    if (bad) {
        std::fprintf(stderr, "%d of %d calls did not reach the launch\n", bad, calls);
        return 1;
    }
    std::printf("layer launch check ok (%d calls)\n", calls);
    return 0;
}
