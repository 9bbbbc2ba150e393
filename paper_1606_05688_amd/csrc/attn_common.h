// attn_common.h -- what the attention operators share: element types, strided heads, which keys a row sees.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/znni.h"

namespace znni {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int ATTN_DMAX = 128;        // widest head
constexpr int PAGE = ZNNI_KV8_PAGE;   // tokens of a page of the 8-bit cache

// Heads of tokens in device memory: element (t, h, d) at data[t * token + h * head + d].
template <typename T>
struct Heads {
    T* data;
    long long token, head;
    __device__ T* row(long long t, int h) const { return data + t * token + h * head; }
};

template <typename T, typename S>
static Heads<T> heads_of(const S* s)
{
    return Heads<T>{(T*)s->data, s->token, s->head};
}

// The rule of visibility: a row at position p sees key j if j <= p + right and (j >= p - left or j < sinks).
struct Window {
    int left, right, sinks;
};

// First and last key of the window part, in 64 bits since left and right may be INT_MAX; keys below `lo` are seen if
// they are sinks.  Rows before all keys have hi < 0 and see nothing.
__host__ __device__ inline void window_of(long long p, int nk, const Window& w, int* lo, int* hi)
{
    const long long a = p - w.left, b = p + w.right;
    *lo = a < 0 ? 0 : a > nk ? nk : (int)a;
    *hi = b < -1 ? -1 : b > nk - 1 ? nk - 1 : (int)b;
}

__host__ __device__ inline bool sees(long long p, int j, const Window& w)
{
    return j <= p + w.right && (j >= p - w.left || j < w.sinks);
}

// A dimension of a launch has fewer than 2^32 threads: workgroups (of up to 256) past this many go on in the second dimension.
constexpr unsigned LAUNCH_X = 1u << 23;
static inline dim3 launch_of(long long groups)
{
    const unsigned x = groups < LAUNCH_X ? (unsigned)groups : LAUNCH_X;
    return dim3(x, (unsigned)((groups + x - 1) / x));
}
__device__ inline long long group_id() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// Host-side checks that the operators share.
static inline bool type_ok(int type) { return type == ZNNI_F32 || type == ZNNI_BF16 || type == ZNNI_F16; }
static inline int type_size(int type) { return type == ZNNI_F32 ? 4 : 2; }

// Rows of heads are read 16 bytes at a time.
static inline bool heads_aligned(const znni_heads* h, int type)
{
    const long long per = 16 / type_size(type);
    return !((uintptr_t)h->data & 15u) && h->token % per == 0 && h->head % per == 0;
}

static inline znni_status heads_shape(int Hq, int Hk, int D)
{
    if (Hq < 1 || Hk < 1 || Hq % Hk || D < 1) return ZNNI_ERR_SHAPE;
    if (Hq > 65535) return ZNNI_ERR_SHAPE;
    if (D % 8 || D > ATTN_DMAX) return ZNNI_ERR_UNSUPPORTED_SIZE;
    return ZNNI_OK;
}

}  // namespace znni
