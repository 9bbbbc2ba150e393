// rows_common.h -- what operators on rows of channels share: their checks, sums over many rows.
#pragma once
#include "attn_common.h"

namespace znni {

constexpr int ROWS_MOST = 1 << 30, COLS_MOST = 1 << 26;

static inline size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// N elements that begin anywhere an element may: one access, which the hardware takes at any address (16 bytes apart it is the faster).
template <typename T, int N>
struct Loose {
    typedef T V __attribute__((ext_vector_type(N)));
    typedef T Anywhere __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    __device__ static V load(const T* p) { return *(const Anywhere*)p; }
    __device__ static void store(T* p, V y) { *(Anywhere*)p = y; }
    // Those of them that are there, zeros for others.
    __device__ static V load(const T* p, int there)
    {
        if (there >= N) return load(p);
        V y;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = e < there ? p[e] : (T)0.f;
        return y;
    }
    __device__ static void store(T* p, V y, int there)
    {
        if (there >= N) {
            store(p, y);
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < there) p[e] = y[e];
    }
};

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

// Sums of `parts` rows of n sums: 32 columns from `col0` on, LANES lanes a column, four reads of a lane on their way at once.
template <typename T, int LANES>
__device__ inline void sum_parts(int n, int parts, const float* __restrict__ sums, T* __restrict__ out, int col0, float (*part)[LANES + 1])
{
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, col = col0 + c;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (col < n)
        for (int i = r; i < parts; i += 4 * LANES)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += i + LANES * j < parts ? sums[(long long)(i + LANES * j) * n + col] : 0.f;
    part[c][r] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    // a column's sums by as many lanes of a wave
    const int mine = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    float y = part[mine][lane];
#pragma unroll
    for (int x = LANES / 2; x; x >>= 1) y += __shfl_xor(y, x, LANES);
    if (lane == 0 && col0 + mine < n) out[col0 + mine] = (T)y;
}

// blockIdx.y: which of the outputs.
template <typename T>
struct SumOut {
    T* to[3];
    const float* from[3];
};

template <typename T>
__global__ __launch_bounds__(1024) void k_sum_parts(int n, int parts, SumOut<T> o)
{
    __shared__ float part[32][33];
    sum_parts<T, 32>(n, parts, o.from[blockIdx.y], o.to[blockIdx.y], (int)blockIdx.x * 32, part);
}

template <typename T>
static znni_status launch_sum_parts(int n, int parts, const SumOut<T>& o, int outputs, hipStream_t st)
{
    k_sum_parts<T><<<dim3((unsigned)((n + 31LL) / 32), (unsigned)outputs), dim3(1024), 0, st>>>(n, parts, o);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni
