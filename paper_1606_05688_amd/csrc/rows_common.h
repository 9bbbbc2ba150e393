// rows_common.h -- what operators on rows of channels share: their checks, sums over many rows.
#pragma once
#include "attn_common.h"

namespace znni {

constexpr int ROWS_MOST = 1 << 30, COLS_MOST = 1 << 26;

static inline size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Whether rows are aligned to `bytes`.
static inline bool rows_wide(const void* p, long long row, int size, int bytes)
{
    return !((uintptr_t)p % bytes) && row * size % bytes == 0;
}

// Tensors that have elements have addresses, aligned to an element; rows that are written do not overlap.
static inline znni_status rows_fine(const znni_rows* r, int type, int rows, int cols, bool written)
{
    if (rows == 0 || cols == 0) return ZNNI_OK;
    if (!r->data) return ZNNI_ERR_NULL;
    if ((uintptr_t)r->data % type_size(type)) return ZNNI_ERR_ALIGN;
    if (written && rows > 1 && r->row < cols) return ZNNI_ERR_SHAPE;
    return ZNNI_OK;
}

// Sums of `parts` rows of n sums, eight lanes a column.  blockIdx.y: which of the outputs.
template <typename T>
struct SumOut {
    T* to[3];
    const float* from[3];
};

template <typename T>
__global__ __launch_bounds__(256) void k_sum_parts(int n, int parts, SumOut<T> o)
{
    __shared__ float part[8][32];
    T* const out = o.to[blockIdx.y];
    const float* const sums = o.from[blockIdx.y];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, col = (int)blockIdx.x * 32 + c;
    float s = 0.f;
    if (col < n)
        for (int i = r; i < parts; i += 8) s += sums[(long long)i * n + col];
    part[r][c] = s;
    __syncthreads();
    if (r || col >= n) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) s += part[q][c];
    out[col] = (T)s;
}

template <typename T>
static znni_status launch_sum_parts(int n, int parts, const SumOut<T>& o, int outputs, hipStream_t st)
{
    k_sum_parts<T><<<dim3((unsigned)((n + 31LL) / 32), (unsigned)outputs), dim3(256), 0, st>>>(n, parts, o);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni
