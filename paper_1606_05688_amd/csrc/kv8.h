// kv8.h -- the 8-bit cache: pages of PAGE tokens, keys [page][head][token][D], values [page][head][D][token], e4m3 codes,
// a power of two for each page, head and kind as scale.
#pragma once
#include "attn_common.h"

namespace znni {

typedef float f32x2 __attribute__((ext_vector_type(2)));

static inline bool cache_aligned(const unsigned char* k, const unsigned char* v, const float* scales)
{
    return !(((uintptr_t)k | (uintptr_t)v) & 15u) && !((uintptr_t)scales & 7u);
}

}  // namespace znni
