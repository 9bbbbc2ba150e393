// kv8_attn.hip -- attention of the last tokens of sequences over the 8-bit cache.
//
// Bound by memory: every code of a visible page is read once.  A wave has sixteen rows (a token's heads that share a key
// and value head, and the tokens after it) and walks pages of its own; eight waves of a workgroup take turns in a part of
// the pages, several workgroups share a sequence, a second kernel joins their parts.  Per page, on 16x16x32 products:
//   scores^T [64 keys][16 rows] = K Q^T, keys ordered so that a lane's 16 scores of its row are 16 keys that follow each
//   other: then the weights are the right operand of  out^T [D][16 rows] = V^T W^T  as they stand, and V^T's operand is
//   16 codes of one element of the head, a load of 16 bytes from pages that keep the tokens innermost.  Nothing goes
//   through LDS before the waves join.
// Codes become bf16 (exact: 4 significant bits); queries and weights are sums of as many bf16 as their type has bits
// for, so products are exact and only sums round, in fp32.
// bf16, 32 sequences of 131072 tokens, heads 32 of 8 x 128, 8.6 GB: 1400 us, 6.1 TB/s, where a large copy reaches 6.25; a window of 4096 in
// 64 sequences, heads 16 of 4 x 128, 267 MB: 46 us, 5.8 TB/s; 777 tokens of one sequence: 8.7 us, the chain length, page, codes, products, join.
#include "attn_join.h"
#include "kv8.h"

namespace znni {

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Kv8Args {
    int Lq, Hq, Hk, D, pages, width, splits;
    const unsigned char* kcodes;
    const unsigned char* vcodes;
    const float* scales;
    const int* table;
    const int* lens;
    Window w;
    float scale;
    float* parts;        // [B][Hk][row tile][splits][16 rows][D]
    float2* stats;       // [B][Hk][row tile][splits][16 rows]: maximum (in powers of two) and sum of weights
};

constexpr int KV8_WAVES = 8, KV8_ROWS = 16;

// bf16 terms that hold a query (exactly) and a weight (to the type's last bit and more)
template <typename T> struct Terms;
template <> struct Terms<bf16> { static constexpr int q = 1, w = 2; };
template <> struct Terms<f16> { static constexpr int q = 2, w = 2; };
template <> struct Terms<float> { static constexpr int q = 3, w = 3; };

// x as N terms: all but the last cut off after eight bits, so that what is left is exact and nothing overflows
template <int N>
__device__ inline void split(float x, bf16* t)
{
#pragma unroll
    for (int n = 0; n < N - 1; ++n) {
        const unsigned h = __float_as_uint(x) >> 16;
        t[n] = __builtin_bit_cast(bf16, (unsigned short)h);
        x -= __uint_as_float(h << 16);
    }
    t[N - 1] = (bf16)x;
}

__device__ inline bf16x8 eight(unsigned a, unsigned b)
{
    bf16x8 r;
    bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    r[0] = x[0]; r[1] = x[1]; r[2] = y[0]; r[3] = y[1];
    r[4] = z[0]; r[5] = z[1]; r[6] = w[0]; r[7] = w[1];
    return r;
}

// The pages of a row tile, in order: those that hold only sinks, then those of the window.
struct Visit {
    int sink_pages, first, n;
    __device__ int index(int i) const { return i < sink_pages ? i : first + i - sink_pages; }
};

__device__ inline Visit visit_of(long long p0, long long p1, int nk, const Window& w)
{
    int lo, hi, a, b;
    window_of(p0, nk, w, &lo, &a);
    window_of(p1, nk, w, &b, &hi);
    Visit v;
    v.first = lo / PAGE;
    const int sinks = min(w.sinks, hi + 1);
    v.sink_pages = min((sinks + PAGE - 1) / PAGE, v.first);
    v.n = hi < lo ? v.sink_pages : v.sink_pages + hi / PAGE - v.first + 1;
    return v;
}

// Steps of 32 elements of a head: lane quarter u has eight of them, in steps that pair up 16 where a load has 16 bytes.
template <int NC, bool FULL>
__device__ inline int element(int c, int u)
{
    return FULL && c < NC / 2 * 2 ? 64 * (c / 2) + 16 * u + 8 * (c % 2) : 32 * c + 8 * u;
}

template <int NC, bool FULL>
__device__ inline void load_keys(const unsigned char* page, int D, int l, uint2 (&k)[4][NC])
{
    const int m = l & 15, u = l >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const unsigned char* row = page + (16 * (m >> 2) + 4 * t + (m & 3)) * D;
        if constexpr (FULL) {
#pragma unroll
            for (int h = 0; h < NC / 2; ++h) {
                const uint4 x = *(const uint4*)(row + 64 * h + 16 * u);
                k[t][2 * h] = make_uint2(x.x, x.y);
                k[t][2 * h + 1] = make_uint2(x.z, x.w);
            }
            if constexpr (NC % 2) k[t][NC - 1] = *(const uint2*)(row + 32 * (NC - 1) + 8 * u);
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) k[t][c] = 32 * c + 8 * u < D ? *(const uint2*)(row + 32 * c + 8 * u) : make_uint2(0, 0);
        }
    }
}

template <int NC, bool FULL>
__device__ inline void load_values(const unsigned char* page, int D, int l, uint4 (&v)[2 * NC])
{
    const int d = l & 15, u = l >> 4;
#pragma unroll
    for (int x = 0; x < 2 * NC; ++x)
        v[x] = FULL || 16 * x + d < D ? *(const uint4*)(page + (16 * x + d) * PAGE + 16 * u) : make_uint4(0, 0, 0, 0);
}

__device__ inline unsigned nan_codes(unsigned x)       // bit 7 of every byte that is NaN (all ones but the sign)
{
    return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

template <typename T, int NC, bool FULL>
__global__ __launch_bounds__(64 * KV8_WAVES) void k_kv8(Kv8Args a, Heads<const T> q, Heads<T> out)
{
    constexpr int NX = 2 * NC, NQ = Terms<T>::q, NW = Terms<T>::w, DP = 32 * NC, LD = DP + 4;
    __shared__ __align__(16) float acc_s[KV8_WAVES][KV8_ROWS][LD];
    __shared__ float top_s[KV8_WAVES][KV8_ROWS], sum_s[KV8_WAVES][KV8_ROWS];
    const int G = a.Hq / a.Hk, tiles = (a.Lq * G + KV8_ROWS - 1) / KV8_ROWS;
    // the row tiles of one part of the pages read the same codes: eight workgroups apart they are on the same XCD at the same time
    // (8 queries of 4 heads, two tiles, 32 sequences of 8192 tokens: 67 us, tile by tile 87)
    int b = blockIdx.z, hk = blockIdx.y, tile = 0, split_id = blockIdx.x;
    if (tiles > 1) {
        const unsigned parts = (unsigned)a.splits * a.Hk * gridDim.z, id = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
        const unsigned in_eights = parts / 8 * 8, rest = parts - in_eights, behind = id - in_eights * tiles;
        const unsigned part_id = id < in_eights * tiles ? id / (8 * tiles) * 8 + id % 8 : in_eights + behind % rest;
        tile = (int)(id < in_eights * tiles ? id / 8 % tiles : behind / rest);
        split_id = (int)(part_id % a.splits);
        hk = (int)(part_id / a.splits % a.Hk);
        b = (int)(part_id / a.splits / a.Hk);
    }
    const int l = threadIdx.x & 63, wave = threadIdx.x >> 6, r = l & 15, u = l >> 4;
    const int len = max(0, (int)min((long long)a.lens[b], (long long)a.width * PAGE));
    const int row = tile * KV8_ROWS + r, rows = a.Lq * G;
    const long long base = (long long)len - a.Lq;
    const long long pos = row < rows ? base + row / G : -1;                                        // of this lane's row
    const long long p0 = base + tile * KV8_ROWS / G, p1 = base + min(tile * KV8_ROWS + KV8_ROWS - 1, rows - 1) / G;
    const Visit visit = visit_of(p0, p1, len, a.w);
    // this workgroup's part of the pages, this wave's turns in it
    const int per = (visit.n + a.splits - 1) / a.splits, end = min(visit.n, (split_id + 1) * per);
    int it = split_id * per + wave;

    bf16x8 qf[NQ][NC];
    {
        const T* p = q.row((long long)b * a.Lq + min(row, rows - 1) / G, hk * G + min(row, rows - 1) % G);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = element<NC, FULL>(c, u);
            T x[8];
            if (FULL || d < a.D) {
#pragma unroll
                for (int n = 0; n < (int)sizeof(T) * 8 / 16; ++n) ((uint4*)x)[n] = ((const uint4*)(p + d))[n];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = (T)0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                bf16 t[NQ];
                split<NQ>((float)x[e], t);
                const bool inf = isinf((float)x[e]);              // which leaves no rest
#pragma unroll
                for (int n = 0; n < NQ; ++n) qf[n][c][e] = n && inf ? (bf16)0.f : t[n];
            }
        }
    }

    f32x4 acc[NX];
#pragma unroll
    for (int x = 0; x < NX; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, sum = 0.f;
    const float by = a.scale * 1.44269504088896340736f;
    const int* table = a.table + (long long)b * a.width;

    // the next page of this wave that exists
    auto next = [&](int i, int* page) {
        for (; i < end; i += KV8_WAVES) {
            *page = __builtin_amdgcn_readfirstlane(table[visit.index(i)]);
            if (*page >= 0 && *page < a.pages) return i;
        }
        return i;
    };
    int page = 0;
    it = __builtin_amdgcn_readfirstlane(next(it, &page));
    uint2 kr[4][NC];
    uint4 vr[NX];
    float2 sc = {0.f, 0.f};
    if (it < end) {
        const long long at = (long long)page * a.Hk + hk;
        load_keys<NC, FULL>(a.kcodes + at * PAGE * a.D, a.D, l, kr);
        load_values<NC, FULL>(a.vcodes + at * PAGE * a.D, a.D, l, vr);
        sc = *(const float2*)(a.scales + at * 2);
    }
    while (it < end) {
        const int key0 = visit.index(it) * PAGE;
        const long long here = (long long)page * a.Hk + hk;
        const float2 s2 = sc;
        int page2 = 0;
        const int it2 = __builtin_amdgcn_readfirstlane(next(it + KV8_WAVES, &page2));
        const long long at = (long long)page2 * a.Hk + hk;

        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const bf16x8 k = eight(kr[t][c].x, kr[t][c].y);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[n][c], s[t], 0, 0, 0);
            }
        }
        if (it2 < end) {
            load_keys<NC, FULL>(a.kcodes + at * PAGE * a.D, a.D, l, kr);
            sc = *(const float2*)(a.scales + at * 2);
        }
        const float c = by * s2.x;
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] *= c;
        // a page that some row sees in part
        const bool whole = key0 + PAGE - 1 <= p0 && (key0 >= p1 - a.w.left || key0 + PAGE <= a.w.sinks);
        bool bad = false;
        if (!whole) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!sees(pos, key0 + 16 * u + 4 * t + i, a.w)) s[t][i] = -INFINITY;
            // values of keys that no row sees count for nothing, whatever they are; NaN that only some rows see are taken
            // out here and given to those rows below
            unsigned keep[4] = {0, 0, 0, 0}, nan = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = key0 + 16 * u + i;
                if (key <= p1 && (key >= p0 - a.w.left || key < a.w.sinks)) keep[i / 4] |= 255u << (8 * (i % 4));
            }
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                unsigned* w = (unsigned*)&vr[x];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] &= keep[i];
                    const unsigned n = nan_codes(w[i]);
                    w[i] &= ~((n >> 7) * 255u);
                    nan |= n;
                }
            }
            bad = __any(nan != 0);
        }
        float t4[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) t4[t] = fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3]));
        float mx = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (__any(mx > top)) {
            const float now = fmaxf(top, mx), old = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
            sum *= old;
#pragma unroll
            for (int x = 0; x < NX; ++x) acc[x] *= old;
            top = now;
        }
        const float zero = top == -INFINITY ? 0.f : top;
        bf16x8 wf[NW][2];
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(s[t][i] - zero);
                part[i] += p;
                bf16 w[NW];
                split<NW>(p * s2.y, w);
#pragma unroll
                for (int n = 0; n < NW; ++n) wf[n][t / 2][(t & 1) * 4 + i] = w[n];
            }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
        for (int x = 0; x < NX; ++x) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 v = h ? eight(vr[x].z, vr[x].w) : eight(vr[x].x, vr[x].y);
#pragma unroll
                for (int n = 0; n < NW; ++n) acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, wf[n][h], acc[x], 0, 0, 0);
            }
        }
        if (it2 < end) load_values<NC, FULL>(a.vcodes + at * PAGE * a.D, a.D, l, vr);
        if (bad) {
            const unsigned char* vp = a.vcodes + here * PAGE * a.D;
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = 16 * x + 4 * u + i;
                    for (int j = 0; j < PAGE && d < a.D; ++j)
                        if ((vp[d * PAGE + j] & 127) == 127 && sees(pos, key0 + j, a.w)) acc[x][i] = NAN;
                }
        }
        it = it2;
        page = page2;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the waves' parts of a row
    if (u == 0) { top_s[wave][r] = top; sum_s[wave][r] = sum; }
#pragma unroll
    for (int x = 0; x < NX; ++x) *(f32x4*)&acc_s[wave][r][16 * x + 4 * u] = acc[x];
    __syncthreads();
    const long long block = (((long long)b * a.Hk + hk) * tiles + tile) * a.splits + split_id;
    for (int i = threadIdx.x; i < KV8_ROWS * DP; i += 64 * KV8_WAVES) {
        const int rr = i / DP, d = i % DP, row_r = tile * KV8_ROWS + rr;
        if (row_r >= rows || d >= a.D) continue;
        float m = -INFINITY, n = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < KV8_WAVES; ++w) m = fmaxf(m, top_s[w][rr]);
        const float z = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < KV8_WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(top_s[w][rr] - z);
            n += f * sum_s[w][rr];
            o += f * acc_s[w][rr][d];
        }
        if (a.splits == 1) {
            out.row((long long)b * a.Lq + row_r / G, hk * G + row_r % G)[d] = (T)(n == 0.f ? 0.f : o / n);
        } else {
            a.parts[(block * KV8_ROWS + rr) * a.D + d] = o;
            if (d == 0) a.stats[block * KV8_ROWS + rr] = make_float2(m, n);
        }
    }
}

// How many workgroups share a sequence's pages.  A call whose waves have two pages at most is not split, which saves the
// launch that joins (13 pages of 4 heads: 8.7 against 10.1 us).  Else a workgroup for every compute unit, none with less than a page a wave
// (16 heads of 47 pages: 24.6 us unsplit, 15.0 split), and more of them where sequences are long, since lengths may differ (64
// sequences of up to 16384 tokens: 128 us unsplit, 116 in four; 64 of 8192 each 100 and 106).
static int kv8_splits(int B, int Lq, int Hq, int Hk, int max_len, int left, int sinks)
{
    const long long tiles = ((long long)Lq * (Hq / Hk) + KV8_ROWS - 1) / KV8_ROWS, groups = tiles * Hk * B;
    const long long seen = (long long)left + Lq < max_len ? (long long)left + Lq + (sinks < max_len ? sinks : max_len) : max_len;
    const long long pages = ((seen < max_len ? seen : max_len) + PAGE - 1) / PAGE;
    if (pages <= 2 * KV8_WAVES) return 1;
    const long long fill = (256 + groups - 1) / groups, most = (pages + KV8_WAVES - 1) / KV8_WAVES;
    const long long even = pages / 64 < 1024 / groups ? pages / 64 : 1024 / groups;
    const long long n = fill > even ? fill : even;
    return (int)(n < most ? n : most);
}

static size_t kv8_part_rows(int B, int Lq, int Hq, int Hk, int splits)
{
    const size_t tiles = ((size_t)Lq * (Hq / Hk) + KV8_ROWS - 1) / KV8_ROWS;
    return splits == 1 ? 0 : tiles * Hk * B * splits * KV8_ROWS;
}

template <typename T, int NC>
static void launch_steps(const Kv8Args& a, dim3 grid, Heads<const T> q, Heads<T> out, hipStream_t st)
{
    if (a.D == 32 * NC) k_kv8<T, NC, true><<<grid, dim3(64 * KV8_WAVES), 0, st>>>(a, q, out);
    else k_kv8<T, NC, false><<<grid, dim3(64 * KV8_WAVES), 0, st>>>(a, q, out);
}

template <typename T>
static znni_status launch_kv8(const Kv8Args& a, int B, const znni_heads* q, const znni_heads* out, hipStream_t st)
{
    const long long rows = (long long)a.Lq * (a.Hq / a.Hk), tiles = (rows + KV8_ROWS - 1) / KV8_ROWS;
    const dim3 grid((unsigned)a.splits, (unsigned)(tiles * a.Hk), (unsigned)B);
    const Heads<const T> qi = heads_of<const T>(q);
    const Heads<T> o = heads_of<T>(out);
    switch ((a.D + 31) / 32) {
        case 1: launch_steps<T, 1>(a, grid, qi, o, st); break;
        case 2: launch_steps<T, 2>(a, grid, qi, o, st); break;
        case 3: launch_steps<T, 3>(a, grid, qi, o, st); break;
        default: launch_steps<T, 4>(a, grid, qi, o, st); break;
    }
    if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
    if (a.splits == 1) return ZNNI_OK;
    const JoinArgs j = {a.Hq, a.Hk, a.D, a.splits, (int)tiles, KV8_ROWS, (int)rows, nullptr, a.Lq, 1.f, a.parts, a.stats};
    return launch_join<T>(j, B, o, st);
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_kv8_attn_workspace(int type, int B, int Lq, int Hq, int Hk, int D, int max_len, int left, int sinks, size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (B < 0 || B > 65535 || Lq < 0 || max_len < 0 || left < 0 || sinks < 0) return ZNNI_ERR_SHAPE;
    const znni_status rc = heads_shape(Hq, Hk, D);
    if (rc) return rc;
    // row tiles of all heads ride in a launch dimension
    if (((long long)Lq * (Hq / Hk) + KV8_ROWS - 1) / KV8_ROWS * Hk > 65535) return ZNNI_ERR_SHAPE;
    *bytes = B && Lq ? kv8_part_rows(B, Lq, Hq, Hk, kv8_splits(B, Lq, Hq, Hk, max_len, left, sinks)) * (D + 2) * sizeof(float) : 0;
    return ZNNI_OK;
}

znni_status znni_kv8_attn(int type, int B, int Lq, int Hq, int Hk, int D, const znni_heads* q, const unsigned char* kcodes,
                          const unsigned char* vcodes, const float* scales, int pages, const int* table, int width,
                          const int* lens, int max_len, int left, int sinks, float scale, const znni_heads* out, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    if (!q || !out) return ZNNI_ERR_NULL;
    size_t need = 0;
    const znni_status rc = znni_kv8_attn_workspace(type, B, Lq, Hq, Hk, D, max_len, left, sinks, &need);
    if (rc) return rc;
    if (pages < 0 || width < 0) return ZNNI_ERR_SHAPE;
    if (B == 0 || Lq == 0) return ZNNI_OK;
    if (!q->data || !out->data || !lens || (need && !workspace)) return ZNNI_ERR_NULL;
    if (pages > 0 && width > 0 && (!kcodes || !vcodes || !scales || !table)) return ZNNI_ERR_NULL;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    if (!heads_aligned(q, type) || !heads_aligned(out, type) || !cache_aligned(kcodes, vcodes, scales) ||
        (((uintptr_t)lens | (uintptr_t)table) & 3u) || (need && ((uintptr_t)workspace & 255u)))
        return ZNNI_ERR_ALIGN;
    const int splits = kv8_splits(B, Lq, Hq, Hk, max_len, left, sinks);
    float* parts = (float*)workspace;
    // (without pages no entry of the table is one: it is not read, and may be NULL)
    const Kv8Args a = {Lq, Hq, Hk, D, pages, pages ? width : 0, splits, kcodes, vcodes, scales, table, lens, {left, 0, sinks}, scale, parts,
                       (float2*)(parts + kv8_part_rows(B, Lq, Hq, Hk, splits) * D)};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_kv8<float>(a, B, q, out, st);
        case ZNNI_BF16: return launch_kv8<bf16>(a, B, q, out, st);
        default: return launch_kv8<f16>(a, B, q, out, st);
    }
}

}  // extern "C"
