// Memory and undefined-behaviour check of the projection operators' host code (test infrastructure), in two builds:
//  - with LAUNCHERS_STAND_IN: the entry points (lq_proj_api.hip, host pass only) under AddressSanitizer and
//    UndefinedBehaviorSanitizer, with launchers that only count: valid calls reach them, every rejection does not;
//  - without: the entry points with their launchers under UndefinedBehaviorSanitizer, up to the launch itself, which fails for
//    want of a GPU.
// Pointers are plain addresses, never dereferenced.
#include <cstdint>
#include <cstdio>

#include "leapquant.h"
#include "lq_internal.hpp"

namespace {
int launches = 0, failures = 0;
void expect(bool ok, const char *what, int line) {
    if (!ok) {
        std::fprintf(stderr, "line %d: %s\n", line, what);
        ++failures;
    }
}
#define EXPECT(c) expect((c), #c, __LINE__)
}  // namespace

namespace lq {
hipError_t launch_decode(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_commit(const lq_dims &, const StatePtrs &, const TokenPtrs &, hipStream_t) { return hipSuccess; }
hipError_t launch_tile(const lq_dims &, const StatePtrs &, int, const float *, float *, const int32_t *, hipStream_t) { return hipSuccess; }
hipError_t launch_baseline(const lq_dims &, void *, int, const TokenPtrs &, hipStream_t) { return hipSuccess; }
#ifdef LAUNCHERS_STAND_IN
hipError_t launch_add_norm(const lq_add &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_gate_norm(const lq_gated &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_quantize_weight(const lq_weight &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_matmul(const lq_matmul &, hipStream_t) { ++launches; return hipSuccess; }
constexpr int32_t REACHED = LQ_OK;
#else
constexpr int32_t REACHED = LQ_EHIP;
#endif
}  // namespace lq

namespace {

template <typename T>
T *P(uintptr_t a = 0x10000) { return reinterpret_cast<T *>(a); }

lq_add add() {
    lq_add a = {};
    a.tokens = 3;
    a.channels = 256;
    a.norm = LQ_NORM_RMS;
    a.out_dtype = LQ_TOKEN_E4M3;
    a.x_stride = a.residual_stride = a.residual_out_stride = a.out_stride = 256;
    a.scale_stride = 2;
    a.x = a.residual = P<void>();
    a.weight = P<float>();
    a.residual_out = a.out = P<void>();
    a.scale = P<float>();
    return a;
}
lq_gated gated(int d = 128) {
    lq_gated g = {};
    g.tokens = 3;
    g.heads = 3;
    g.d = d;
    g.out_dtype = LQ_TOKEN_E4M3;
    g.x_stride = g.gate_stride = g.out_stride = 3 * d;
    g.scale_stride = (3 * d + 127) / 128;
    g.x = g.gate = P<void>();
    g.weight = P<float>();
    g.out = P<void>();
    g.scale = P<float>();
    return g;
}
lq_weight weight() {
    lq_weight w = {};
    w.n = 200;
    w.k = 256;
    w.w_stride = w.out_stride = 256;
    w.w = P<void>();
    w.out = P<void>();
    w.scale = P<float>();
    return w;
}
lq_matmul product(int64_t tokens = 3, int32_t n = 200, int32_t k = 256) {
    lq_matmul m = {};
    m.tokens = tokens;
    m.n = n;
    m.k = k;
    m.x_stride = m.w_stride = k;
    m.x_scale_stride = (k + 127) / 128;
    m.out_stride = (n + 7) / 8 * 8;
    m.x = m.w = P<void>();
    m.x_scale = m.w_scale = P<float>();
    m.out = P<void>();
    return m;
}

void valid_calls() {
    const int32_t R = lq::REACHED;
    for (int32_t channels : {8, 512, 1024, 2048, 4096, 8192, 16384})
        for (int64_t tokens : {(int64_t)1, (int64_t)3, (int64_t)INT32_MAX}) {
            lq_add a = add();
            a.tokens = tokens;
            a.channels = channels;
            a.x_stride = a.residual_stride = a.residual_out_stride = a.out_stride = 1LL << 30;
            a.scale_stride = 1LL << 30;
            EXPECT(leapquant_add_norm(&a, nullptr) == R);
        }
    for (int32_t d : {64, 128, 256, 384, 16384}) {
        lq_gated g = gated(d);
        EXPECT(leapquant_gate_norm(&g, nullptr) == R);
        g.tokens = INT32_MAX;
        g.heads = 1 << 20;
        g.x_stride = g.gate_stride = g.out_stride = g.scale_stride = 1LL << 40;
        EXPECT(leapquant_gate_norm(&g, nullptr) == R);
    }
    // strides that nobody has to set: of one row, and of arrays that are not there
    for (int64_t stride : {INT64_MAX, INT64_MIN, (int64_t)0}) {
        lq_add a = add();
        a.tokens = 1;
        a.x_stride = a.residual_stride = a.residual_out_stride = a.out_stride = a.scale_stride = stride;
        EXPECT(leapquant_add_norm(&a, nullptr) == R);
        a = add();
        a.residual = nullptr;
        a.residual_out = nullptr;
        a.residual_stride = a.residual_out_stride = stride;
        a.out_dtype = LQ_TOKEN_BF16;
        a.scale = nullptr;
        a.scale_stride = stride;
        EXPECT(leapquant_add_norm(&a, nullptr) == R);
        lq_gated g = gated();
        g.tokens = 1;
        g.x_stride = g.gate_stride = g.out_stride = g.scale_stride = stride;
        EXPECT(leapquant_gate_norm(&g, nullptr) == R);
        lq_weight w = weight();
        w.n = 1;
        w.w_stride = w.out_stride = stride;
        EXPECT(leapquant_quantize_weight(&w, nullptr) == R);
        lq_matmul m = product(1, 1);
        m.x_stride = m.x_scale_stride = m.w_stride = m.out_stride = stride;
        EXPECT(leapquant_matmul(&m, nullptr) == R);
    }
    // every rule of the product's sizes, both types
    for (int32_t type : {LQ_TOKEN_F32, LQ_TOKEN_BF16})
        for (int64_t tokens : {(int64_t)1, (int64_t)4, (int64_t)5, (int64_t)32, (int64_t)33, (int64_t)300, (int64_t)8192, (int64_t)1 << 20, (int64_t)1 << 28})
            for (int32_t n : {1, 64, 1000, 12288, 1 << 26})
                for (int32_t k : {16, 128, 4096, 1 << 12}) {
                    lq_matmul m = product(tokens, n, k);
                    m.out_dtype = type;
                    const bool fits = tokens <= (1LL << 36) / n;
                    EXPECT(leapquant_matmul(&m, nullptr) == (fits ? R : LQ_EUNSUPPORTED));
                }
    lq_matmul m = product(1 << 28, 1, 1 << 23);
    EXPECT(leapquant_matmul(&m, nullptr) == R);
    m.tokens += 1;
    EXPECT(leapquant_matmul(&m, nullptr) == LQ_EUNSUPPORTED);
    m = product(2, 1 << 13, 1 << 23);
    EXPECT(leapquant_matmul(&m, nullptr) == R);
    lq_weight w = weight();
    EXPECT(leapquant_quantize_weight(&w, nullptr) == R);
    w.n = INT32_MAX;
    w.k = 112;
    w.w_stride = w.out_stride = 1LL << 40;
    EXPECT(leapquant_quantize_weight(&w, nullptr) == LQ_EUNSUPPORTED);      // (2^24 blocks)
    w.n = INT32_MAX - 256;
    EXPECT(leapquant_quantize_weight(&w, nullptr) == R);
}

void rejections() {
    const int before = launches;
    for (int i = 0; i < 14; ++i) {
        lq_add a = add();
        switch (i) {
            case 0: a.tokens = INT64_MAX; break;
            case 1: a.tokens = INT64_MIN; break;
            case 2: a.channels = INT32_MAX; break;
            case 3: a.channels = INT32_MIN; break;
            case 4: a.x_stride = INT64_MAX; break;
            case 5: a.residual_stride = INT64_MIN; break;
            case 6: a.scale_stride = INT64_MAX; break;
            case 7: a.norm = INT32_MAX; break;
            case 8: a.out_dtype = INT32_MIN; break;
            case 9: a.eps = -1.0f; break;
            case 10: a.scale = P<float>(0x10002); break;
            case 11: a.residual_out = P<void>(0x10008); break;
            case 12: a.weight = P<float>(0x10004); break;
            default: a.x = nullptr; break;
        }
        EXPECT(leapquant_add_norm(&a, nullptr) < 0);
    }
    for (int i = 0; i < 10; ++i) {
        lq_gated g = gated();
        switch (i) {
            case 0: g.tokens = INT64_MAX; break;
            case 1: g.heads = INT32_MAX; break;
            case 2: g.d = INT32_MAX; break;
            case 3: g.d = INT32_MIN; break;
            case 4: g.x_stride = INT64_MAX; break;
            case 5: g.scale_stride = INT64_MIN; break;
            case 6: g.act = INT32_MAX; break;
            case 7: g.gate_first = INT32_MIN; break;
            case 8: g.heads = 0; break;
            default: g.gate = P<void>(0x10001); break;
        }
        EXPECT(leapquant_gate_norm(&g, nullptr) < 0);
    }
    for (int i = 0; i < 6; ++i) {
        lq_weight w = weight();
        switch (i) {
            case 0: w.n = INT32_MIN; break;
            case 1: w.k = INT32_MAX; break;
            case 2: w.n = INT32_MAX; w.k = INT32_MAX - 15; break;
            case 3: w.w_stride = INT64_MAX; break;
            case 4: w.out_stride = INT64_MIN; break;
            default: w.dtype = INT32_MAX; break;
        }
        EXPECT(leapquant_quantize_weight(&w, nullptr) < 0);
    }
    for (int i = 0; i < 14; ++i) {
        lq_matmul m = product();
        switch (i) {
            case 0: m.tokens = INT64_MAX; break;
            case 1: m.tokens = INT64_MIN; break;
            case 2: m.n = INT32_MAX; break;
            case 3: m.k = INT32_MAX - 15; break;
            case 4: m.k = INT32_MIN; break;
            case 5: m.x_stride = INT64_MAX; break;
            case 6: m.w_stride = INT64_MIN; break;
            case 7: m.out_stride = INT64_MAX; break;
            case 8: m.x_scale_stride = INT64_MAX; break;
            case 9: m.out_dtype = LQ_TOKEN_E4M3; break;
            case 10: m.tokens = INT32_MAX; m.n = 1 << 26; break;
            case 11: m.bias = P<float>(0x10002); break;
            case 12: m.w = nullptr; break;
            default: m.n = 1 << 26; m.k = 1 << 22; m.w_stride = m.x_stride = 1 << 22; m.x_scale_stride = 1 << 15; m.out_stride = 1 << 26; break;
        }
        EXPECT(leapquant_matmul(&m, nullptr) < 0);
    }
    EXPECT(launches == before);
}

}  // namespace

int main() {
#ifndef LAUNCHERS_STAND_IN
    int n = 0;
    if (hipGetDeviceCount(&n) == hipSuccess && n > 0) {
        std::printf("a GPU is visible: nothing is launched\n");
        return 1;
    }
#endif
    valid_calls();
    rejections();
    if (failures) {
        std::fprintf(stderr, "%d failures\n", failures);
        return 1;
    }
    std::printf("projection check ok\n");
    return 0;
}
