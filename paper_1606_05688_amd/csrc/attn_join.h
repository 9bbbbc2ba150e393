// attn_join.h -- joins the parts of rows whose keys were split over workgroups.
#pragma once
#include "attn_common.h"

namespace znni {

// Part s of row r (of a batch entry and key head) of `rows` lies at ((bh * tiles + r / tile_rows) * splits + s) * tile_rows
// + r % tile_rows: D weighted sums of values, and their maximum (in powers of two) and sum of weights in `stats`.
struct JoinArgs {
    int Hq, Hk, D, splits, tiles, tile_rows, rows;
    const int* cu;              // starts of the sequences' queries; NULL: all have `queries`
    int queries;
    const float* parts;
    const float2* stats;
};

// One wave a row, elements over its lanes.
template <typename T>
__global__ __launch_bounds__(256) void k_join(JoinArgs a, long long all, Heads<T> out)
{
    const int G = a.Hq / a.Hk, l = threadIdx.x & 63;
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= all) return;
    const int row = (int)(id % a.rows);
    const long long bh = id / a.rows;
    const int hk = (int)(bh % a.Hk), b = (int)(bh / a.Hk);
    const long long token = a.cu ? a.cu[b] : (long long)b * a.queries;
    if (a.cu && row / G >= a.cu[b + 1] - a.cu[b]) return;
    const long long first = (bh * a.tiles + row / a.tile_rows) * a.splits * a.tile_rows + row % a.tile_rows;
    float m = -INFINITY;
    for (int s = l; s < a.splits; s += 64) m = fmaxf(m, a.stats[first + (long long)s * a.tile_rows].x);
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float z = m == -INFINITY ? 0.f : m;
    float n = 0.f, o0 = 0.f, o1 = 0.f;
    for (int s = 0; s < a.splits; ++s) {
        const long long at = first + (long long)s * a.tile_rows;
        const float2 st = a.stats[at];
        const float f = __builtin_amdgcn_exp2f(st.x - z);
        n += f * st.y;
        if (l < a.D) o0 += f * a.parts[at * a.D + l];
        if (l + 64 < a.D) o1 += f * a.parts[at * a.D + l + 64];
    }
    T* y = out.row(token + row / G, hk * G + row % G);
    if (l < a.D) y[l] = (T)(n == 0.f ? 0.f : o0 / n);
    if (l + 64 < a.D) y[l + 64] = (T)(n == 0.f ? 0.f : o1 / n);
}

template <typename T>
static znni_status launch_join(const JoinArgs& a, int B, Heads<T> out, hipStream_t st)
{
    const long long all = (long long)a.rows * a.Hk * B;
    k_join<T><<<dim3((unsigned)((all + 3) / 4)), dim3(256), 0, st>>>(a, all, out);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni
