// attn_join.h -- joins the parts of rows whose keys were split over workgroups.
#pragma once
#include "attn_common.h"

namespace znni {

// Part s of row r (of a batch entry and key head) of `rows` lies at ((bh * tiles + r / tile_rows) * splits + s) * tile_rows
// + r % tile_rows: D weighted sums of values, and their maximum (`by` times that in powers of two) and sum of weights in `stats`.
struct JoinArgs {
    int Hq, Hk, D, splits, tiles, tile_rows, rows;
    const int* cu;              // starts of the sequences' queries; NULL: all have `queries`
    int queries;
    float by;
    const float* parts;
    const float2* stats;
};

// The row, its token and head, and where its first part is; false past the sequence's end.
struct JoinRow {
    long long token, first;
    int head;
    __device__ bool find(const JoinArgs& a, unsigned id)
    {
        const int G = a.Hq / a.Hk, row = (int)(id % (unsigned)a.rows);
        const unsigned bh = id / (unsigned)a.rows;
        const int hk = (int)(bh % (unsigned)a.Hk), b = (int)(bh / (unsigned)a.Hk);
        token = (a.cu ? a.cu[b] : (long long)b * a.queries) + row / G;
        head = hk * G + row % G;
        first = ((long long)bh * a.tiles + row / a.tile_rows) * a.splits * a.tile_rows + row % a.tile_rows;
        return !a.cu || row / G < a.cu[b + 1] - a.cu[b];
    }
};

// A part's sum times the part's factor.  An infinite one stays so: the row sees an infinity, and a factor that rounds to zero would make NaN of it.
__device__ inline float share_of(float f, float sum) { return fabsf(sum) == INFINITY ? sum : f * sum; }

constexpr int JOIN_FEW = 8;          // parts that a lane reads at once

// Few parts: LANES lanes a row, four elements a lane, everything read at once (13720 rows of 4 parts of 40 elements, 9 MB: 4.4 us, a wave
// a row 10.2, four waves a row 24).
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_join_few(JoinArgs a, unsigned all, Heads<T> out)
{
    const unsigned id = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int d = threadIdx.x % LANES * 4;
    JoinRow r;
    if (id >= all || d >= a.D || !r.find(a, id)) return;
    float2 st[JOIN_FEW];
    float4 p[JOIN_FEW];
#pragma unroll
    for (int i = 0; i < JOIN_FEW; ++i)
        if (i < a.splits) {
            const long long at = r.first + (long long)i * a.tile_rows;
            st[i] = a.stats[at];
            p[i] = *(const float4*)(a.parts + at * a.D + d);
        }
    float m = -INFINITY, n = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN_FEW; ++i)
        if (i < a.splits) m = fmaxf(m, st[i].x);
    const float z = m == -INFINITY ? 0.f : m;
    float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_FEW; ++i)
        if (i < a.splits) {
            const float f = __builtin_amdgcn_exp2f((st[i].x - z) * a.by);
            n += f * st[i].y;
            o.x += share_of(f, p[i].x);
            o.y += share_of(f, p[i].y);
            o.z += share_of(f, p[i].z);
            o.w += share_of(f, p[i].w);
        }
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 y = {(T)0.f, (T)0.f, (T)0.f, (T)0.f};
    if (n != 0.f) y = T4{(T)(o.x / n), (T)(o.y / n), (T)(o.z / n), (T)(o.w / n)};
    *(T4*)(out.row(r.token, r.head) + d) = y;
}

// Many parts: four waves a row take turns in them, a lane has two elements.  Bound by the chain of reads (maxima, then parts): four
// parts of a wave are on their way together (128 rows of 16 parts of 128 elements: 4 us, a wave a row 13).
template <typename T>
__global__ __launch_bounds__(256) void k_join(JoinArgs a, Heads<T> out)
{
    __shared__ float2 acc_s[4][ATTN_DMAX / 2];
    __shared__ float sum_s[4];
    const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
    JoinRow r;
    if (!r.find(a, blockIdx.x)) return;
    float m = -INFINITY;
    for (int s = l; s < a.splits; s += 64) m = fmaxf(m, a.stats[r.first + (long long)s * a.tile_rows].x);
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float z = m == -INFINITY ? 0.f : m;
    const int d = min(2 * l, a.D - 2);
    float n = 0.f;
    float2 o = {0.f, 0.f};
    for (int s0 = wave; s0 < a.splits; s0 += 16) {
        float2 st[4], p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long at = r.first + (long long)min(s0 + 4 * i, a.splits - 1) * a.tile_rows;
            st[i] = a.stats[at];
            p[i] = *(const float2*)(a.parts + at * a.D + d);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (s0 + 4 * i >= a.splits) break;
            const float f = __builtin_amdgcn_exp2f((st[i].x - z) * a.by);
            n += f * st[i].y;
            o.x += share_of(f, p[i].x);
            o.y += share_of(f, p[i].y);
        }
    }
    acc_s[wave][l] = o;
    if (l == 0) sum_s[wave] = n;
    __syncthreads();
    if (wave || 2 * l >= a.D) return;
    n = (sum_s[0] + sum_s[1]) + (sum_s[2] + sum_s[3]);
    o.x = (acc_s[0][l].x + acc_s[1][l].x) + (acc_s[2][l].x + acc_s[3][l].x);
    o.y = (acc_s[0][l].y + acc_s[1][l].y) + (acc_s[2][l].y + acc_s[3][l].y);
    typedef T T2 __attribute__((ext_vector_type(2)));
    T2 y;
    y[0] = (T)(n == 0.f ? 0.f : o.x / n);
    y[1] = (T)(n == 0.f ? 0.f : o.y / n);
    *(T2*)(out.row(r.token, r.head) + d) = y;
}

template <typename T>
static znni_status launch_join(const JoinArgs& a, int B, Heads<T> out, hipStream_t st)
{
    const unsigned all = (unsigned)((long long)a.rows * a.Hk * B);
    if (a.splits > JOIN_FEW) k_join<T><<<dim3(all), dim3(256), 0, st>>>(a, out);
    else if (a.D <= 64) k_join_few<T, 16><<<dim3((all + 15) / 16), dim3(256), 0, st>>>(a, all, out);
    else k_join_few<T, 32><<<dim3((all + 7) / 8), dim3(256), 0, st>>>(a, all, out);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni
