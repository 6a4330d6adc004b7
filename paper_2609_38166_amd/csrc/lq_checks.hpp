// Host checks of arguments that the C entry points of the layer and projection operators share.
#pragma once

#include <stdint.h>

#include "leapquant.h"

namespace lq {

// a launch's work-items are counted in 32 bits: workgroups of 256
constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;

inline bool flag(int32_t x) { return x == 0 || x == 1; }
inline bool token_type(int32_t x) { return x == LQ_TOKEN_F32 || x == LQ_TOKEN_BF16; }
inline int64_t token_size(int32_t t) { return t == LQ_TOKEN_BF16 ? 2 : 4; }

// A required (or optional: may be NULL) pointer with an alignment.
inline int32_t check(const void *p, uintptr_t n, bool needed = true) {
    if (!p) return needed ? LQ_EINVAL : LQ_OK;
    return (uintptr_t)p & (n - 1) ? LQ_EALIGN : LQ_OK;
}

// A token array: rows of `row` elements of `size` bytes, `stride` elements apart.
inline int32_t check_rows(const void *p, int64_t tokens, int64_t row, int64_t stride, int64_t size, uintptr_t align) {
    if (tokens == 0) return LQ_OK;
    const int32_t e = check(p, align);
    if (e != LQ_OK) return e;
    if (tokens > 1) {
        if (stride < row || stride > (1LL << 40)) return LQ_EINVAL;
        if (stride * size % (int64_t)align) return LQ_EALIGN;
    }
    return LQ_OK;
}

// cu_seqlens entries, slots and positions are 32-bit.
inline int32_t check_tokens(int64_t tokens) {
    if (tokens < 0) return LQ_EINVAL;
    return tokens > INT32_MAX ? LQ_EUNSUPPORTED : LQ_OK;
}

}  // namespace lq
