// Short causal convolution per channel, prompts (packed sequences) and single
// tokens:  y[t][c] = act(bias[c] + sum_i w[c][K-1-i] x[t-i][c]).
//
// Bound: HBM; K multiply-adds per value read.  A thread owns 16 bytes of
// channels of a run of tokens, whose input rows it reads once into registers;
// neighbouring lanes own neighbouring channels, so every access is whole lines.
// 8192 tokens x 8192 channels, bf16, K = 4: 62 us (a large copy's rate: 56); a wave that
// walks one run only 65-70.  256 tokens x 12288 channels 12.1 us (11.9).
#include <algorithm>

#include "lq_layer.hpp"
#include "lq_internal.hpp"

namespace lq {

namespace {

constexpr int RUN = 8;      // tokens that a wave has in registers at a time

struct ConvArgs {
    const char *x;
    const float *weight, *bias;
    char *out;
    char *state;
    const int32_t *cu, *slots;
    int32_t *err;
    int64_t tokens, x_stride, out_stride;      // strides in bytes
    int32_t seqs, channels, n_slots, silu, carry, blocks_c, blocks_t, runs;
};

template <int K, bool BF>
__device__ __forceinline__ void load_params(const ConvArgs &a, int c, float (*w)[K], float *bias) {
    constexpr int V = Tok<BF>::V;
    float flat[V * K];
#pragma unroll
    for (int i = 0; i < V * K / 4; ++i) {
        const float4 p = ((const float4 *)(a.weight + (int64_t)c * K))[i];
        flat[4 * i] = p.x; flat[4 * i + 1] = p.y; flat[4 * i + 2] = p.z; flat[4 * i + 3] = p.w;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int j = 0; j < K; ++j) w[v][j] = flat[v * K + j];
        bias[v] = a.bias ? a.bias[c + v] : 0.0f;
    }
}

// Output of one token from its K input rows (oldest first).
template <int K, bool BF, bool OBF>
__device__ __forceinline__ void emit(const ConvArgs &a, char *to, const uint4 *rows, const float (*w)[K], const float *bias) {
    constexpr int V = Tok<BF>::V;
    float y[V];
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = bias[v];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        float f[V];
        unpack16<BF>(rows[j], f);
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] = fmaf(w[v][j], f[v], y[v]);
    }
    if (a.silu) {
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] *= __builtin_amdgcn_rcpf(1.0f + __expf(-y[v]));
    }
    store_tok<OBF, V>(to, y);
}

__device__ __forceinline__ uint4 fill16(uint32_t w) { return make_uint4(w, w, w, w); }

// Row `i` (0 oldest) of what precedes a sequence: its state, zero, or NaN.
template <int K, bool BF>
__device__ __forceinline__ uint4 old_row(const ConvArgs &a, int slot, int i, int64_t c_bytes) {
    if (slot == BAD_SLOT) return fill16(BF ? 0x7FC07FC0u : 0x7FC00000u);
    if (!a.carry || slot == NO_SLOT) return fill16(0u);
    return *(const uint4 *)(a.state + ((int64_t)slot * (K - 1) + i) * a.channels * Tok<BF>::BYTES + c_bytes);
}

// Last sequence that begins at or before token t (-1: none), over the seqs
// entries of cu; the whole wave searches, 64 entries at a time.
__device__ __forceinline__ int find_sequence(const int32_t *cu, int seqs, int64_t t, int lane) {
    int lo = 0, hi = seqs;                       // the count of entries <= t lies in [lo, hi]
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const int p = __popcll(__ballot(at < hi && cu[at < hi ? at : lo] <= t));
        if (p == 0) return lo - 1;
        hi = min(hi, lo + p * step);
        lo = lo + (p - 1) * step + 1;
    }
    const int at = lo + lane;
    return lo + __popcll(__ballot(at < hi && cu[at < hi ? at : 0] <= t)) - 1;
}

// The first K-1 tokens of a sequence, whose windows reach its start, and its new state,
// from memory (inputs past the sequence's end do not count).
template <int K, bool BF, bool OBF>
__device__ __forceinline__ void begin_sequence(const ConvArgs &a, Span s, int slot, int64_t c_bytes, const float (*w)[K],
                                            const float *bias, int c) {
    const int64_t n = s.end - s.begin;
    uint4 line[2 * (K - 1)], keep[K - 1];       // the old state's rows, then the first inputs
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        line[j] = old_row<K, BF>(a, slot, j, c_bytes);
        line[K - 1 + j] = *(const uint4 *)(a.x + (s.begin + (j < n ? j : 0)) * a.x_stride + c_bytes);
        const int64_t at = n - (K - 1) + j;     // place in the sequence of the new state's row j
        keep[j] = at >= 0 ? *(const uint4 *)(a.x + (s.begin + at) * a.x_stride + c_bytes)
                          : old_row<K, BF>(a, slot, (int)(K - 1 + at), c_bytes);
    }
#pragma unroll
    for (int j = 0; j < K - 1; ++j)
        if (j < n) emit<K, BF, OBF>(a, a.out + (s.begin + j) * a.out_stride + (int64_t)c * Tok<OBF>::BYTES, line + j, w, bias);
    if (slot >= 0) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
            *(uint4 *)(a.state + ((int64_t)slot * (K - 1) + j) * a.channels * Tok<BF>::BYTES + c_bytes) = keep[j];
    }
}

// One wave: the channels of its 64 lanes, a.runs times RUN tokens one after the other,
// the next RUN rows on their way meanwhile.  The first K-1 tokens of a sequence read the
// old state and its last K-1 replace it in place, so the wave that holds a sequence's
// first token computes all of those K-1 tokens (also past its own) and then writes the
// new state: nobody else reads the old one.
template <int K, bool BF, bool OBF>
__global__ __launch_bounds__(256) void conv_prompt_kernel(ConvArgs a) {
    constexpr int V = Tok<BF>::V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x / a.blocks_c;
    const int c = ((int)(blockIdx.x - block * a.blocks_c) * 64 + lane) * V;
    const bool here = c < a.channels;
    const int64_t cb = (int64_t)(here ? c : 0) * Tok<BF>::BYTES;

    if (blockIdx.x == 0) {
        check_seqlens(a.cu, a.seqs, a.tokens, a.err, threadIdx.x, 256);
        // (slots of empty sequences, whose states nobody looks at below)
        if (a.err && a.carry)
            for (int b = threadIdx.x; b < a.seqs; b += 256) state_row(a.state, a.slots, b, a.n_slots, a.err);
    }
    if (block >= a.blocks_t) {
        // empty sequences without carry: their state becomes zero
        if (a.carry) return;
        const int b = (block - a.blocks_t) * 4 + wave;
        if (b >= a.seqs) return;
        const Span s = sequence_span(a.cu, b, a.tokens);
        const int slot = state_row(a.state, a.slots, b, a.n_slots, a.err);
        if (s.begin == s.end && slot >= 0 && here) {
#pragma unroll
            for (int i = 0; i < K - 1; ++i)
                *(uint4 *)(a.state + ((int64_t)slot * (K - 1) + i) * a.channels * Tok<BF>::BYTES + cb) = fill16(0u);
        }
        return;
    }

    const int64_t first = ((int64_t)block * 4 + wave) * (RUN * a.runs);
    if (first >= a.tokens) return;
    const int64_t last = min(first + RUN * a.runs, a.tokens);
    const char *xc = a.x + cb;
    uint4 rows[K - 1 + RUN], next[RUN];         // input rows t0 - (K-1) .. t0 + RUN - 1, and the RUN after them
#pragma unroll
    for (int i = 0; i < K - 1 + RUN; ++i) {
        const int64_t t = min(max(first - (K - 1) + i, (int64_t)0), a.tokens - 1);
        rows[i] = *(const uint4 *)(xc + t * a.x_stride);
    }
    float w[V][K], bias[V];
    load_params<K, BF>(a, here ? c : 0, w, bias);

    const int first_b = find_sequence(a.cu, a.seqs, first, lane);
    int b = first_b;
    Span s{0, 0};
    int64_t following = a.tokens;               // the next sequence's first token
    auto enter = [&]() {
        if (b >= 0) s = sequence_span(a.cu, b, a.tokens);
        following = b + 1 < a.seqs ? (int64_t)a.cu[b + 1] : a.tokens;
    };
    enter();
    for (int64_t t0 = first; t0 < last; t0 += RUN) {
        if (t0 + RUN < last) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) next[i] = *(const uint4 *)(xc + min(t0 + RUN + i, a.tokens - 1) * a.x_stride);
        }
        char *to = a.out + t0 * a.out_stride + (int64_t)c * Tok<OBF>::BYTES;
        if (b >= 0 && t0 - s.begin >= K - 1 && t0 + RUN <= s.end) {
            // all of it inside one sequence, past its start
            if (here) {
#pragma unroll
                for (int i = 0; i < RUN; ++i) emit<K, BF, OBF>(a, to + i * a.out_stride, rows + i, w, bias);
            }
        } else {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                const int64_t t = t0 + i;
                if (t >= last) break;
                while (t >= following && b + 1 < a.seqs) {
                    ++b;
                    enter();
                }
                if (b < 0 || t >= s.end || t < s.begin) continue;      // belongs to no sequence
                if (t - s.begin >= K - 1 && here) emit<K, BF, OBF>(a, to + i * a.out_stride, rows + i, w, bias);
            }
        }
#pragma unroll
        for (int i = 0; i < K - 1; ++i) rows[i] = rows[RUN + i];
#pragma unroll
        for (int i = 0; i < RUN; ++i) rows[K - 1 + i] = next[i];
    }
    // the sequences that begin here
    for (b = max(first_b, 0); b < a.seqs && a.cu[b] < last; ++b) {
        s = sequence_span(a.cu, b, a.tokens);
        if (s.begin < first || s.begin == s.end) continue;
        const int slot = state_row(a.state, a.slots, b, a.n_slots, a.err);
        if (here) begin_sequence<K, BF, OBF>(a, s, slot, cb, w, bias, c);
    }
}

// R requests per thread: the channels' weights are read once for them.
template <int K, bool BF, bool OBF, int R>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvArgs a) {
    constexpr int V = Tok<BF>::V;
    const int first = blockIdx.x / a.blocks_c;
    const int c = ((int)(blockIdx.x - first * a.blocks_c) * 256 + (int)threadIdx.x) * V;
    if (c >= a.channels) return;
    const int64_t cb = (int64_t)c * Tok<BF>::BYTES;
    uint4 rows[R][K];
    int slot[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int b = min(first * R + r, a.seqs - 1);
        slot[r] = first * R + r < a.seqs ? state_row(a.state, a.slots, b, a.n_slots, a.err) : NO_SLOT;
        rows[r][K - 1] = *(const uint4 *)(a.x + (int64_t)b * a.x_stride + cb);
#pragma unroll
        for (int i = 0; i < K - 1; ++i) rows[r][i] = old_row<K, BF>(a, slot[r], i, cb);
    }
    float w[V][K], bias[V];
    load_params<K, BF>(a, c, w, bias);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int b = first * R + r;
        if (b >= a.seqs) break;
        if (slot[r] >= 0) {
#pragma unroll
            for (int i = 0; i < K - 1; ++i)
                *(uint4 *)(a.state + ((int64_t)slot[r] * (K - 1) + i) * a.channels * Tok<BF>::BYTES + cb) = rows[r][i + 1];
        }
        emit<K, BF, OBF>(a, a.out + (int64_t)b * a.out_stride + (int64_t)c * Tok<OBF>::BYTES, rows[r], w, bias);
    }
}

ConvArgs conv_args(const lq_conv &c) {
    ConvArgs a;
    a.x = (const char *)c.x;
    a.weight = c.weight;
    a.bias = c.bias;
    a.out = (char *)c.out;
    a.state = (char *)c.state;
    a.cu = c.cu_seqlens;
    a.slots = c.slots;
    a.err = c.err;
    a.tokens = c.tokens;
    a.x_stride = row_bytes(c.tokens, c.x_stride, c.dtype == LQ_TOKEN_BF16 ? 2 : 4);
    a.out_stride = row_bytes(c.tokens, c.out_stride, c.out_dtype == LQ_TOKEN_BF16 ? 2 : 4);
    a.seqs = c.seqs;
    a.channels = c.channels;
    a.n_slots = c.n_slots;
    a.silu = c.silu;
    a.carry = c.carry;
    a.runs = 1;
    a.blocks_c = a.blocks_t = 0;
    return a;
}

template <int K, bool BF, bool OBF>
hipError_t launch(ConvArgs a, bool step, hipStream_t st) {
    const int per = (step ? 256 : 64) * Tok<BF>::V;
    a.blocks_c = (a.channels + per - 1) / per;
    if (step) {
        a.carry = 1;
        // Four requests per thread where the launch fills the GPU all the same, us a call (1, 2,
        // 4; bf16, width 4, fp32 out): 256 x 12288 14.8, 12.4, 12.2; 128 x 12288 9.1, 8.5, 8.0;
        // 64 x 8192 4.5, 4.9, 6.1.
        const int64_t single = (int64_t)a.blocks_c * a.seqs;
        if (single >= 512)
            hipLaunchKernelGGL((conv_step_kernel<K, BF, OBF, 4>), dim3(a.blocks_c * ((a.seqs + 3) / 4)), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((conv_step_kernel<K, BF, OBF, 1>), dim3((unsigned)single), dim3(256), 0, st, a);
    } else {
        // Runs per wave: as few as leave one round of workgroups (512: their registers allow
        // two per CU), up to eight; a launch of several rounds anyway takes two.  us, each
        // timed by itself in one go: 131 tokens x 1536 fp32 channels 5.3, 6.5, 14.0 with 1, 2, 8;
        // 2048 x 8192 bf16 20, 17, 19, 20 with 1, 2 (the rule's), 3, 4; 3000 x 6144 bf16 22, 21, 19,
        // 22, 26 with 1, 2, 3 (the rule's), 4, 8; 8192 x 8192 bf16 65, 59, 60, 62, 62, 61, 67, 57
        // with 1 .. 8 (eight: exactly one round), 75 with 16; 32768 x 12288 bf16 354, 304, 302,
        // 309 with 1, 2, 4, 8.  Not so good: 4096 x 8192 fp32 51, 60, 53, 56, 57, 57, 59, 61 with 1 .. 8.
        const int64_t groups = (a.tokens + 4 * RUN - 1) / (4 * RUN), round = std::max(512 / a.blocks_c, 1);
        const int64_t runs = std::max<int64_t>((groups + round - 1) / round, 1);
        a.runs = runs > 8 ? 2 : (int)runs;
        a.blocks_t = (int)((a.tokens + 4 * RUN * a.runs - 1) / (4 * RUN * a.runs));
        int extra = a.state && !a.carry ? (a.seqs + 3) / 4 : 0;
        if (a.blocks_t + extra == 0) {
            if (!a.err) return hipSuccess;
            extra = 1;                          // no tokens: the lengths are checked all the same
        }
        hipLaunchKernelGGL((conv_prompt_kernel<K, BF, OBF>), dim3(a.blocks_c * (a.blocks_t + extra)), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

template <int K>
hipError_t launch_types(const lq_conv &c, bool step, hipStream_t st) {
    const ConvArgs a = conv_args(c);
    const bool obf = c.out_dtype == LQ_TOKEN_BF16;
    if (c.dtype == LQ_TOKEN_BF16)
        return obf ? launch<K, true, true>(a, step, st) : launch<K, true, false>(a, step, st);
    return obf ? launch<K, false, true>(a, step, st) : launch<K, false, false>(a, step, st);
}

hipError_t launch_width(const lq_conv &c, bool step, hipStream_t st) {
    switch (c.width) {
        case 2: return launch_types<2>(c, step, st);
        case 3: return launch_types<3>(c, step, st);
        default: return launch_types<4>(c, step, st);
    }
}

}  // namespace

hipError_t launch_conv_prompt(const lq_conv &c, hipStream_t st) { return launch_width(c, false, st); }
hipError_t launch_conv_step(const lq_conv &c, hipStream_t st) { return launch_width(c, true, st); }

}  // namespace lq
