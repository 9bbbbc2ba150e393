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

// WAVES waves a row (1 or 4) take turns in its parts, a lane has two elements.  Bound by the chain of reads (maxima, then parts): four
// parts of a wave are on their way together.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void k_join(JoinArgs a, unsigned all, Heads<T> out)
{
    __shared__ float2 acc_s[4][ATTN_DMAX / 2];
    __shared__ float sum_s[4];
    const int G = a.Hq / a.Hk, l = threadIdx.x & 63, wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
    const unsigned id = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (id >= all) return;
    const int row = (int)(id % (unsigned)a.rows);
    const unsigned bh = id / (unsigned)a.rows;
    const int hk = (int)(bh % (unsigned)a.Hk), b = (int)(bh / (unsigned)a.Hk);
    const long long token = a.cu ? a.cu[b] : (long long)b * a.queries;
    if (a.cu && row / G >= a.cu[b + 1] - a.cu[b]) return;
    const long long first = ((long long)bh * a.tiles + row / a.tile_rows) * a.splits * a.tile_rows + row % a.tile_rows;
    float m = -INFINITY;
    for (int s = l; s < a.splits; s += 64) m = fmaxf(m, a.stats[first + (long long)s * a.tile_rows].x);
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float z = m == -INFINITY ? 0.f : m;
    const int d = min(2 * l, a.D - 2);
    float n = 0.f;
    float2 o = {0.f, 0.f};
    for (int s0 = wave; s0 < a.splits; s0 += 4 * WAVES) {
        float2 st[4], p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long at = first + (long long)min(s0 + WAVES * i, a.splits - 1) * a.tile_rows;
            st[i] = a.stats[at];
            p[i] = *(const float2*)(a.parts + at * a.D + d);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (s0 + WAVES * i >= a.splits) break;
            const float f = __builtin_amdgcn_exp2f(st[i].x - z);
            n += f * st[i].y;
            o.x += f * p[i].x;
            o.y += f * p[i].y;
        }
    }
    if constexpr (WAVES > 1) {
        acc_s[wave][l] = o;
        if (l == 0) sum_s[wave] = n;
        __syncthreads();
        if (wave) return;
        n = (sum_s[0] + sum_s[1]) + (sum_s[2] + sum_s[3]);
        o.x = (acc_s[0][l].x + acc_s[1][l].x) + (acc_s[2][l].x + acc_s[3][l].x);
        o.y = (acc_s[0][l].y + acc_s[1][l].y) + (acc_s[2][l].y + acc_s[3][l].y);
    }
    if (2 * l >= a.D) return;
    typedef T T2 __attribute__((ext_vector_type(2)));
    T2 y;
    y[0] = (T)(n == 0.f ? 0.f : o.x / n);
    y[1] = (T)(n == 0.f ? 0.f : o.y / n);
    *(T2*)(out.row(token + row / G, hk * G + row % G) + d) = y;
}

template <typename T>
static znni_status launch_join(const JoinArgs& a, int B, Heads<T> out, hipStream_t st)
{
    const long long all = (long long)a.rows * a.Hk * B;
    // 128 rows of 16 parts: 13 us with a wave a row, 4 with four; 13720 rows of 4 parts: 24 us with four waves a row, 10 with one
    if (a.splits > 8) k_join<T, 4><<<dim3((unsigned)all), dim3(256), 0, st>>>(a, (unsigned)all, out);
    else k_join<T, 1><<<dim3((unsigned)((all + 3) / 4)), dim3(256), 0, st>>>(a, (unsigned)all, out);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni
