// linear.hip -- matrix products of tokens with weights: bias, activation and residual where the product ends, and the gradients.
//
//   out[m][n] = residual[m][n] + act(z[m][n]),   z[m][n] = sum_k x[m][k] w[n][k] + bias[n]
//   dz = dout act'(z),   dx[m][k] = sum_n dz[m][n] w[n][k],   dw[n][k] = sum_m dz[m][n] x[m][k],   dbias[n] = sum_m dz[m][n]
//
// Three products, whose sums run along the contiguous index of both operands, of one, of none.  Large ones are bound by the matrix instructions and the
// LDS reads that feed them: 256 x 256 of the result a workgroup, eight waves of 128 x 64 (six operands read for eight products of 32 x 32), steps of 64 in
// two buffers by direct loads, reads ahead of products, neighbouring tiles on one XCD.  bf16 8192^3: 840 to 940 us by card (1170 to 1310
// TFLOP/s; a library's product on one of these cards 1415), 4096^3 1100 to 1210 TFLOP/s, 32768 x 2048 x 8192 1000 (the 537 MB of results go out while no product
// runs: a workgroup that brought the next tile first waited for its own stores, 1215 us against 1160).  Tiles of 32 steps in four buffers: 12 % slower.
// fp32 135 TFLOP/s of 157.  Up to 32 rows: bound by the weights, which go from memory straight into registers (8 x 2048 x 4096 bf16: 5.7 us, 2.9 TB/s).
// The gradients' dz is made once, with its sums over tokens: bound by memory (13824 x 4096 bf16, gelu: 68 us, 5 TB/s; with a branching erfc 148).
#include <type_traits>

#include "product_tile.h"
#include "rows_common.h"

namespace znni {

// ---- activations ----------------------------------------------------------------------------------------------------

// The normal distribution up to z, and e^(-z^2/2).  Below zero it is e^(-z^2/2) t P(t), t = 1 / (1 + p |z|): P fitted to erfcx, which has no
// steep part, with a relative error of 9e-8 up to |z| = 14; so the tail, where 1 + erf has no bits left, keeps its own.
__device__ inline float normal_up_to(float z, float* bell)
{
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170368f * z * z), t = __builtin_amdgcn_rcpf(fmaf(0.23333333333f, fabsf(z), 1.f));
    float p = fmaf(t, -0.0677811997f, 0.230613793f);
    p = fmaf(t, p, -0.176407345f);
    p = fmaf(t, p, 0.205008941f);
    p = fmaf(t, p, 0.0232055263f);
    p = fmaf(t, p, 0.100732062f);
    p = fmaf(t, p, 0.0914526451f);
    p = fmaf(t, p, 0.0931755651f);
    const float tail = e * t * p;
    *bell = e;
    return z > 0.f ? 1.f - tail : tail;
}
__device__ inline float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z)); }

template <int ACT>
__device__ inline float activated(float z)
{
    float bell;
    if constexpr (ACT == ZNNI_ACT_RELU) return z < 0.f ? 0.f : z;            // (NaN stays)
    if constexpr (ACT == ZNNI_ACT_GELU) return z * normal_up_to(z, &bell);
    if constexpr (ACT == ZNNI_ACT_SILU) return z * logistic(z);
    return z;
}

template <int ACT>
__device__ inline float slope(float z)
{
    if constexpr (ACT == ZNNI_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
    if constexpr (ACT == ZNNI_ACT_GELU) {
        float bell;
        const float up = normal_up_to(z, &bell);
        return fmaf(z * 0.39894228040143267794f, bell, up);
    }
    if constexpr (ACT == ZNNI_ACT_SILU) {
        const float p = logistic(z);
        return p * fmaf(z, 1.f - p, 1.f);
    }
    return 1.f;
}

template <typename F>
static auto with_act(int act, F f)
{
    switch (act) {
        case ZNNI_ACT_RELU: return f(std::integral_constant<int, ZNNI_ACT_RELU>());
        case ZNNI_ACT_GELU: return f(std::integral_constant<int, ZNNI_ACT_GELU>());
        case ZNNI_ACT_SILU: return f(std::integral_constant<int, ZNNI_ACT_SILU>());
        default: return f(std::integral_constant<int, ZNNI_ACT_NONE>());
    }
}

// ---- where a product ends -------------------------------------------------------------------------------------------

template <typename T>
struct End {
    const T* bias;
    const T* residual;
    T* z;
    T* out;
    long long residual_row, z_row, out_row;
    float* parts;               // sums of a part of the steps, [split][M][Np], instead of all that
    int Np;
};

// N consecutive elements of a row, as far as they are there.
template <typename T, int ACT, int N>
__device__ inline void end_row(const End<T>& d, long long m, int n, int there, const float* v)
{
    using L = Loose<T, N>;
    typename L::V b, r, z, o;
    if (d.bias) b = L::load(d.bias + n, there);
    if (d.residual) r = L::load(d.residual + m * d.residual_row + n, there);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        float y = v[e];
        if (d.bias) y += (float)b[e];
        z[e] = (T)y;
        y = activated<ACT>(y);
        if (d.residual) y += (float)r[e];
        o[e] = (T)y;
    }
    if (d.z) L::store(d.z + m * d.z_row + n, z, there);
    L::store(d.out + m * d.out_row + n, o, there);
}
template <typename T, int ACT>
__device__ inline void end_four(const End<T>& d, long long m, int n, int there, float4 v)
{
    const float y[4] = {v.x, v.y, v.z, v.w};
    end_row<T, ACT, 4>(d, m, n, there, y);
}

// ---- products over tiles --------------------------------------------------------------------------------------------

struct ProductArgs {
    int M, N, K;
    int tiles_m, tiles_n, splits, per;      // steps of the sum that a split takes
};

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: runs of 32 tiles, eight rows by four columns, to the same one.
__device__ inline void tile_of(int id, int tiles_m, int tiles_n, int* tm, int* tn)
{
    const int n = tiles_m * tiles_n;
    if (id < n / 256 * 256) id = (id / 256 * 8 + id % 8) * 32 + id / 8 % 32;
    const int band = id / (8 * tiles_n), first = band * 8, high = min(8, tiles_m - first), at = id - band * 8 * tiles_n;
    *tm = first + at % high;
    *tn = at / high;
}

// out^T [n][m] += W^T X: the columns of the result are the left operand, so that a lane holds four consecutive columns of a row.
// WAVES_N x WAVES_M waves of NB x MB products of 32 x 32.
template <typename T, bool LI, bool RI, int WAVES_N, int WAVES_M, int NB, int MB, int STAGES>
struct ProductShape {
    static constexpr int THREADS = 64 * WAVES_N * WAVES_M, TN = WAVES_N * NB * 32, TM = WAVES_M * MB * 32;
    using L = Tile<T, LI, TN, THREADS>;
    using R = Tile<T, RI, TM, THREADS>;
    typedef char Tiles[STAGES][L::BYTES + R::BYTES];
};

template <typename T, bool LI, bool RI, int WAVES_N, int WAVES_M, int NB, int MB, int STAGES, int ACT>
__device__ __forceinline__ void product(const ProductArgs& a, const Side<T>& left, const Side<T>& right, const End<T>& d, long long group,
                                        typename ProductShape<T, LI, RI, WAVES_N, WAVES_M, NB, MB, STAGES>::Tiles& tiles)
{
    using S = ProductShape<T, LI, RI, WAVES_N, WAVES_M, NB, MB, STAGES>;
    using L = typename S::L;
    using R = typename S::R;
    using M = Mfma<T>;
    constexpr int TN = S::TN, TM = S::TM;
    long long id = group;
    const int split = (int)(id % a.splits); id /= a.splits;
    int tm, tn;
    tile_of((int)id, a.tiles_m, a.tiles_n, &tm, &tn);
    const int m0 = tm * TM, n0 = tn * TN;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wn = wave % WAVES_N * NB * 32, wm = wave / WAVES_N * MB * 32;
    const int begin = split * a.per, end = min(a.K, begin + a.per);
    const int n = end > begin ? (end - begin + L::BK - 1) / L::BK : 0;
    L lt;
    R rt;
    lt.find(left, n0, t);
    rt.find(right, m0, t);
    auto bring = [&](int it) {
        char* const to = tiles[it % STAGES];
        lt.bring(left, n0, begin + it * L::BK, end, to, t);
        rt.bring(right, m0, begin + it * L::BK, end, to + L::BYTES, t);
    };
    constexpr int ONE = STAGES > 2 ? L::PER + R::PER : 0, TWO = STAGES > 3 ? 2 * ONE : 0;      // loads of tiles behind the present one
    f32x16 acc[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < n) bring(i);
    for (int it = 0; it < n; ++it) {
        // tile `it` is there, those behind it may be on their way
        const int behind = min(STAGES - 2, n - 1 - it);
        if (STAGES > 3 && behind == 2) wait_but_and_meet<TWO>();
        else if (STAGES > 2 && behind == 1) wait_but_and_meet<ONE>();
        else wait_but_and_meet<0>();
        if (it + STAGES - 1 < n) bring(it + STAGES - 1);
        const char* const lb = tiles[it % STAGES];
        const char* const rb = lb + L::BYTES;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            typename M::V x[NB], y[MB];
#pragma unroll
            for (int i = 0; i < NB; ++i) x[i] = L::operand(lb, wn + 32 * i, c, l);
#pragma unroll
            for (int j = 0; j < MB; ++j) y[j] = R::operand(rb, wm + 32 * j, c, l);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) {
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j] = M::mul(x[i][e], y[j][e], acc[i][j]);
                    } else {
                        acc[i][j] = M::mul(x[i], y[j], acc[i][j]);
                    }
                }
        }
        // reads of a step run ahead of the products of the one before
        if constexpr (sizeof(T) == 2) {
            constexpr int READS = NB * (LI ? 1 : 2) + MB * (RI ? 1 : 2), PRODUCTS = NB * MB;
            __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
            for (int i = 0; i < 4 * PRODUCTS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (READS + PRODUCTS - 1) / PRODUCTS, 0);
            }
        }
    }
    const int h = l >> 5, c32 = l & 31;
    if (a.splits > 1) {
#pragma unroll
        for (int j = 0; j < MB; ++j) {
            const int m = m0 + wm + 32 * j + c32;
            if (m >= a.M) continue;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int col = n0 + wn + 32 * i + 8 * q + 4 * h;
                    if (col < a.N)
                        *(float4*)(d.parts + ((long long)split * a.M + m) * d.Np + col) =
                            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
        }
        return;
    }
    // A lane has four columns of a row, 32 rows side by side: through LDS, a wave's 32 rows at a time, they become whole lines of memory.
    // (Chunk c of row r at c ^ r: lanes that write have a row each, lanes that read consecutive chunks.)
    constexpr int EC = 16 / sizeof(T), COLS = 32 * NB, CHUNKS = COLS / 4, LANES = COLS / EC;
    static_assert(WAVES_N * WAVES_M * 32 * COLS * 4 <= STAGES * (L::BYTES + R::BYTES), "a wave's rows fit its part of LDS");
    __syncthreads();
    float4* const mine = (float4*)&tiles[0][0] + wave * 32 * CHUNKS;
#pragma unroll
    for (int j = 0; j < MB; ++j) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[c32 * CHUNKS + ((8 * i + 2 * q + h) ^ (c32 & (CHUNKS - 1)))] =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        wave_meets();
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 64 / LANES) {
            const int r = r0 + l / LANES, c = l % LANES * EC, m = m0 + wm + 32 * j + r, col = n0 + wn + c;
            float4 v[EC / 4];
#pragma unroll
            for (int e = 0; e < EC / 4; ++e) v[e] = mine[r * CHUNKS + ((c / 4 + e) ^ (r & (CHUNKS - 1)))];
            if (m >= a.M || col >= a.N) continue;
            end_row<T, ACT, EC>(d, m, col, a.N - col, (const float*)v);
        }
        wave_meets();
    }
}

template <typename T, bool LI, bool RI, int WAVES_N, int WAVES_M, int NB, int MB, int STAGES, int ACT>
__global__ __launch_bounds__(64 * WAVES_N * WAVES_M, 2) void k_product(ProductArgs a, Side<T> left, Side<T> right, End<T> d)
{
    __shared__ __align__(1024) typename ProductShape<T, LI, RI, WAVES_N, WAVES_M, NB, MB, STAGES>::Tiles tiles;
    const long long group = group_id();
    if (group < (long long)a.tiles_m * a.tiles_n * a.splits) product<T, LI, RI, WAVES_N, WAVES_M, NB, MB, STAGES, ACT>(a, left, right, d, group, tiles);
}

// The gradients of a small layer in one launch, since none waits for another: dx, dw, and the sums of the bias's parts.
template <typename T>
struct Gradients {
    ProductArgs x, w;
    Side<T> x_left, x_right, w_left, w_right;
    End<T> dx, dw;
    int n, parts;
    const float* sums;
    T* dbias;                    // or NULL
};
template <typename T>
__global__ __launch_bounds__(256, 2) void k_gradients(Gradients<T> g)
{
    typedef typename ProductShape<T, false, true, 2, 2, 1, 1, 4>::Tiles Tiles;
    static_assert(sizeof(Tiles) == sizeof(typename ProductShape<T, false, false, 2, 2, 1, 1, 4>::Tiles), "one size for both");
    __shared__ __align__(1024) Tiles tiles;
    const long long group = group_id(), x = (long long)g.x.tiles_m * g.x.tiles_n * g.x.splits, w = (long long)g.w.tiles_m * g.w.tiles_n * g.w.splits;
    if (group < x) product<T, false, true, 2, 2, 1, 1, 4, ZNNI_ACT_NONE>(g.x, g.x_left, g.x_right, g.dx, group, tiles);
    else if (group < x + w) product<T, false, false, 2, 2, 1, 1, 4, ZNNI_ACT_NONE>(g.w, g.w_left, g.w_right, g.dw, group - x, tiles);
    else if (g.dbias && (group - x - w) * 32 < g.n) sum_parts<T, 8>(g.n, g.parts, g.sums, g.dbias, (int)(group - x - w) * 32, *(float(*)[32][9])&tiles);
}

// Sums of the parts of the steps, then what an unsplit product does at its end.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_product_join(int M, int N, int splits, End<T> d)
{
    const long long i = (group_id() * 256 + threadIdx.x) * 4;
    const int n = (int)(i % d.Np);
    const long long m = i / d.Np;
    if (m >= M) return;
    float4 v = {0.f, 0.f, 0.f, 0.f};
    const long long step = (long long)M * d.Np;
    for (int s = 0; s < splits; ++s) {
        const float4 p = *(const float4*)(d.parts + s * step + i);
        v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
    }
    end_four<T, ACT>(d, m, n, N - n, v);
}

// ---- few rows -------------------------------------------------------------------------------------------------------

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ inline f32x4 mul16(Mfma<bf16>::V a, Mfma<bf16>::V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mul16(Mfma<f16>::V a, Mfma<f16>::V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mul16(Mfma<float>::V a, Mfma<float>::V b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

constexpr int FEW_WAVES = 8;

// Up to 16 MB rows: bound by reading the weights.  A workgroup has 16 columns of the result, whose weights its waves read straight into
// registers, each a part of the steps, several loads on their way at once; their sums meet in LDS.
template <typename T, int MB, int ACT>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_few(ProductArgs a, Side<T> w, Side<T> x, End<T> d)
{
    constexpr int EC = 16 / sizeof(T), STEP = 4 * EC, AHEAD = MB == 1 ? 8 : 4;
    typedef typename Mfma<T>::V V;
    __shared__ f32x4 sums[FEW_WAVES][MB][64];
    const long long group = group_id();
    const int split = (int)(group % a.splits), n0 = (int)(group / a.splits) * 16;
    if (n0 >= a.N) return;
    const int l = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = l & 15, c = (l >> 4) * EC;
    const int begin = split * a.per, end = min(a.K, begin + a.per);
    const int mine = ((end - begin + STEP - 1) / STEP + FEW_WAVES - 1) / FEW_WAVES * STEP;
    const int k0 = begin + wave * mine, k1 = min(end, k0 + mine);
    const T* const wp = w.p + (long long)min(n0 + c16, a.N - 1) * w.ld + c;
    const T* xp[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) xp[j] = x.p + (long long)min(16 * j + c16, a.M - 1) * x.ld + c;
    f32x4 acc[MB] = {};
    for (int k = k0; k < k1; k += STEP * AHEAD) {
        V y[AHEAD], z[MB][AHEAD];
        if (k + STEP * AHEAD <= k1) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                y[s] = Loose<T, EC>::load(wp + k + s * STEP);
#pragma unroll
                for (int j = 0; j < MB; ++j) z[j][s] = Loose<T, EC>::load(xp[j] + k + s * STEP);
            }
        } else {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int there = k1 - (k + s * STEP + c);
                y[s] = Loose<T, EC>::load(wp + k + s * STEP, there);
#pragma unroll
                for (int j = 0; j < MB; ++j) z[j][s] = Loose<T, EC>::load(xp[j] + k + s * STEP, there);
            }
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[j] = mul16(y[s], z[j][s], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) sums[wave][j][l] = acc[j];
    __syncthreads();
    if (wave >= MB) return;
    const int m = 16 * wave + c16, n = n0 + 4 * (l >> 4);
    if (m >= a.M || n >= a.N) return;
    f32x4 s = sums[0][wave][l];
#pragma unroll
    for (int i = 1; i < FEW_WAVES; ++i) s += sums[i][wave][l];
    const float4 v = make_float4(s[0], s[1], s[2], s[3]);
    if (a.splits > 1) *(float4*)(d.parts + ((long long)split * a.M + m) * d.Np + n) = v;
    else end_four<T, ACT>(d, m, n, a.N - n, v);
}

constexpr int SPLITS_MOST = 32;
constexpr int FEW = 32;                  // rows that k_few takes

struct ProductPlan {
    int kind;                    // 0: tiles of 64 x 64, 1: 128 x 128, 2: 256 x 256, -1: few rows
    int splits, per;
    size_t parts;                // elements
};

// both_inner: the sum's index is the contiguous one on both sides.
static ProductPlan product_plan(int type, int M, int N, int K, bool both_inner)
{
    ProductPlan p;
    const int bk = type == ZNNI_F32 ? 32 : 64;
    if (both_inner && M <= FEW) {
        // workgroups share the steps while there are fewer than compute units, each wave with 16 loads at least
        p.kind = -1;
        const long long n = ((long long)N + 15) / 16, most = (long long)K / (FEW_WAVES * 16 * (bk / 2));
        long long s = 256 / (n ? n : 1);
        if (s > most) s = most;
        if (s > SPLITS_MOST) s = SPLITS_MOST;
        if (s < 1) s = 1;
        p.per = (int)(((K + s - 1) / s + bk - 1) / bk * bk);
        p.splits = K ? (int)(((long long)K + p.per - 1) / p.per) : 1;
        p.parts = p.splits > 1 ? (size_t)p.splits * M * ((N + 3) / 4 * 4) : 0;
        return p;
    }
    auto tiles = [&](long long e) { return ((M + e - 1) / e) * ((N + e - 1) / e); };
    // Tiles of 256 x 256 have a compute unit each, of 128 x 128 two share one; a round of the latter, half the work, takes 0.57 of the time (8192^3
    // bf16: 864 us and 985).  So whichever fills its last round better: 13824 x 2048 x 4096 (4 rounds, 7 half ones) 242 us and 248, its dw, 2048 x
    // 4096 outputs (1, 1) 300 and 203.  With less than half a round of the smaller tiles, 64 x 64 and the steps split.
    const long long r2 = 100 * ((tiles(256) + 255) / 256), r1 = 57 * ((tiles(128) + 511) / 512);
    p.kind = tiles(128) < 256 ? 0 : type != ZNNI_F32 && r2 <= r1 + r1 / 20 ? 2 : 1;
    const long long n = tiles(64 << p.kind), steps = ((long long)K + bk - 1) / bk;
    // Few tiles: workgroups share the steps, if that saves more than the second launch costs: a step takes 0.6 us (fp32 1.2) where a compute unit has
    // one workgroup, joining the parts 4.5 (bf16, 336 columns, 400 steps of the sum, 1300 rows: 9.3 us with four parts, 6.0 with one); where rows
    // of odd lengths come by way of registers, three times that.
    long long s = p.kind == 0 && n < 256 ? 512 / (n ? n : 1) : 1;
    if (s > steps / 2) s = steps / 2;
    if (s > SPLITS_MOST) s = SPLITS_MOST;
    if (s < 1 || (steps - steps / s) * (type == ZNNI_F32 ? 12 : 6) * (K % (bk / 8) || N % (bk / 8) ? 3 : 1) < 45) s = 1;
    p.per = (int)((steps + s - 1) / s * bk);
    p.splits = K ? (int)(((long long)K + p.per - 1) / p.per) : 1;
    p.parts = p.splits > 1 ? (size_t)p.splits * M * ((N + 3) / 4 * 4) : 0;
    return p;
}

static ProductArgs product_args(const ProductPlan& p, int M, int N, int K)
{
    const int edge = 64 << (p.kind < 0 ? 0 : p.kind);
    return {M, N, K, (int)((M + (long long)edge - 1) / edge), (int)((N + (long long)edge - 1) / edge), p.splits, p.per};
}

template <typename T, int ACT>
static znni_status join_product(const ProductPlan& p, int M, int N, const End<T>& d, hipStream_t st)
{
    if (p.splits == 1) return ZNNI_OK;
    k_product_join<T, ACT><<<launch_of(((long long)M * d.Np / 4 + 255) / 256), dim3(256), 0, st>>>(M, N, p.splits, d);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

template <typename T, bool LI, bool RI, int ACT>
static znni_status launch_product(int M, int N, int K, Side<T> left, Side<T> right, End<T> d, hipStream_t st)
{
    const int type = sizeof(T) == 4 ? ZNNI_F32 : ZNNI_BF16;
    const ProductPlan p = product_plan(type, M, N, K, LI && RI);
    d.Np = (N + 3) / 4 * 4;
    const ProductArgs a = product_args(p, M, N, K);
    const unsigned threads = p.kind == 2 ? 512 : 256;
    const dim3 grid = launch_of((long long)a.tiles_m * a.tiles_n * p.splits, threads);
    if constexpr (LI && RI) {
        if (p.kind < 0) {
            const dim3 few = launch_of((long long)((N + 15) / 16) * p.splits, 64 * FEW_WAVES), block(64 * FEW_WAVES);
            if (M <= 16) k_few<T, 1, ACT><<<few, block, 0, st>>>(a, left, right, d);
            else k_few<T, 2, ACT><<<few, block, 0, st>>>(a, left, right, d);
        }
    }
    if (p.kind == 0) k_product<T, LI, RI, 2, 2, 1, 1, 4, ACT><<<grid, dim3(threads), 0, st>>>(a, left, right, d);
    else if (p.kind == 1) k_product<T, LI, RI, 2, 2, 2, 2, 2, ACT><<<grid, dim3(threads), 0, st>>>(a, left, right, d);
    else if constexpr (sizeof(T) == 2) {
        if (p.kind == 2) k_product<T, LI, RI, 2, 4, 4, 2, 2, ACT><<<grid, dim3(threads), 0, st>>>(a, left, right, d);
    }
    if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
    return join_product<T, ACT>(p, M, N, d, st);
}

// ---- gradient of what went into the activation, sums over tokens ----------------------------------------------------

constexpr int SLOPE_ROWS = 8;             // rows of a workgroup at a time
constexpr int SLOPE_PARTS = 256;          // parts of a sum over all tokens at most

// dz = dout act'(z) (written if there is an activation), and its sum over `per` rows, 32 chunks of columns by 8 rows a workgroup.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_slope(int M, int N, int per, const T* __restrict__ dout, long long dout_row, const T* __restrict__ z,
                                               long long z_row, T* __restrict__ dz, int dz_row, float* __restrict__ sums)
{
    constexpr int VEC = 16 / sizeof(T);
    using L = Loose<T, VEC>;
    __shared__ float part[SLOPE_ROWS][32 * VEC];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, n = ((int)blockIdx.x * 32 + c) * VEC;
    const int m0 = (int)blockIdx.y * per, m1 = (int)min((long long)M, (long long)m0 + per);
    float s[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = 0.f;
    if (n < N)
        for (int m = m0 + r; m < m1; m += SLOPE_ROWS) {
            const typename L::V g = L::load(dout + m * dout_row + n, N - n);
            if constexpr (ACT != ZNNI_ACT_NONE) {
                const typename L::V y = L::load(z + m * z_row + n, N - n);
                typename L::V o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float f = (float)g[e] * slope<ACT>((float)y[e]);
                    s[e] += f;
                    o[e] = (T)f;
                }
                *(typename L::V*)(dz + (long long)m * dz_row + n) = o;           // (rows of dz are padded)
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[e] += (float)g[e];
            }
        }
    if (!sums) return;
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[r][c * VEC + e] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * VEC; i += 256) {
        const int col = (int)blockIdx.x * 32 * VEC + i;
        if (col >= N) break;
        float y = 0.f;
#pragma unroll
        for (int q = 0; q < SLOPE_ROWS; ++q) y += part[q][i];
        sums[(long long)blockIdx.y * N + col] = y;
    }
}

static int slope_parts(int M, int N)
{
    // about 1024 workgroups, of 32 rows at least
    const long long across = ((long long)N + 255) / 256;
    long long n = 1024 / (across > 0 ? across : 1);
    if (n > ((long long)M + 31) / 32) n = ((long long)M + 31) / 32;
    if (n > SLOPE_PARTS) n = SLOPE_PARTS;
    return n < 1 ? 1 : (int)n;
}

// ---- what a call needs ----------------------------------------------------------------------------------------------

struct BackwardPlan {
    size_t dz, sums, parts, more;      // bytes; `more`: parts of dw, where dx and dw are made at once
    int dz_row;
    bool at_once;
    ProductPlan x, w;
    size_t all() const { return dz + sums + parts + more; }
};

static BackwardPlan backward_plan(int type, int M, int N, int K, int act, bool dx, bool dw, bool dbias)
{
    BackwardPlan p = {};
    const int per = 16 / type_size(type);
    p.dz_row = (int)(((long long)N + per - 1) / per * per);
    const bool products = dx || dw;
    if (act != ZNNI_ACT_NONE && (products || dbias)) p.dz = up((size_t)M * p.dz_row * type_size(type));
    if (dbias) p.sums = up((size_t)slope_parts(M, N) * N * sizeof(float));
    p.x = product_plan(type, M, K, N, false);
    p.w = product_plan(type, N, K, M, false);
    size_t parts = dx ? p.x.parts : 0;
    p.at_once = dx && dw && M > 0 && N > 0 && K > 0 && p.x.kind == 0 && p.w.kind == 0;
    if (p.at_once) p.more = up(p.w.parts * sizeof(float));
    else if (dw && p.w.parts > parts) parts = p.w.parts;
    p.parts = up(parts * sizeof(float));
    return p;
}

template <typename T>
static Side<T> side_of(const znni_rows* r, int rows)
{
    return {(const T*)r->data, r->row, rows, rows_wide(r->data, r->row, sizeof(T), 16)};
}

template <typename T>
static End<T> end_of(const znni_rows* out)
{
    End<T> d = {};
    d.out = (T*)out->data;
    d.out_row = out->row;
    return d;
}

template <typename T>
static znni_status forward(int M, int N, int K, const znni_rows* x, const znni_rows* w, const void* bias, int act, const znni_rows* residual,
                           const znni_rows* z, const znni_rows* out, void* workspace, hipStream_t st)
{
    End<T> d = end_of<T>(out);
    d.bias = (const T*)bias;
    if (residual) {
        d.residual = (const T*)residual->data;
        d.residual_row = residual->row;
    }
    if (z) {
        d.z = (T*)z->data;
        d.z_row = z->row;
    }
    d.parts = (float*)workspace;
    return with_act(act, [&](auto k) {
        return launch_product<T, true, true, decltype(k)::value>(M, N, K, side_of<T>(w, N), side_of<T>(x, M), d, st);
    });
}

template <typename T>
static znni_status backward(int type, int M, int N, int K, const znni_rows* dout, const znni_rows* x, const znni_rows* w, const znni_rows* z, int act,
                            const znni_rows* dx, const znni_rows* dw, void* dbias, void* workspace, hipStream_t st)
{
    const BackwardPlan p = backward_plan(type, M, N, K, act, dx, dw, dbias);
    char* at = (char*)workspace;
    T* const dz = (T*)at;
    float* const sums = dbias ? (float*)(at + p.dz) : nullptr;
    float* const parts = (float*)(at + p.dz + p.sums);
    znni_rows g = *dout;
    if (M > 0 && N > 0 && (act != ZNNI_ACT_NONE || dbias)) {
        const int n = slope_parts(M, N), per = (int)(((long long)M + n - 1) / n);
        const T* y = z ? (const T*)z->data : nullptr;
        const long long yr = z ? z->row : 0;
        with_act(act, [&](auto k) {
            constexpr int ACT = decltype(k)::value, across = 32 * 16 / sizeof(T);
            const dim3 grid((unsigned)((N + (long long)across - 1) / across), (unsigned)n);
            k_slope<T, ACT><<<grid, dim3(256), 0, st>>>(M, N, per, (const T*)dout->data, dout->row, y, yr, dz, p.dz_row, sums);
            return 0;
        });
        if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
        if (act != ZNNI_ACT_NONE) g = {dz, p.dz_row};
    }
    if (p.at_once) {
        Gradients<T> y = {};
        y.x = product_args(p.x, M, K, N);
        y.w = product_args(p.w, N, K, M);
        y.x_left = side_of<T>(w, K);
        y.x_right = side_of<T>(&g, M);
        y.w_left = side_of<T>(x, K);
        y.w_right = side_of<T>(&g, N);
        y.dx = end_of<T>(dx);
        y.dw = end_of<T>(dw);
        y.dx.Np = y.dw.Np = (K + 3) / 4 * 4;
        y.dx.parts = parts;
        y.dw.parts = (float*)(at + p.dz + p.sums + p.parts);
        y.n = N;
        y.parts = slope_parts(M, N);
        y.sums = sums;
        y.dbias = (T*)dbias;
        const long long groups = (long long)y.x.tiles_m * y.x.tiles_n * p.x.splits + (long long)y.w.tiles_m * y.w.tiles_n * p.w.splits;
        k_gradients<T><<<launch_of(groups + (dbias ? (N + 31) / 32 : 0)), dim3(256), 0, st>>>(y);
        if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
        const znni_status rc = join_product<T, ZNNI_ACT_NONE>(p.x, M, K, y.dx, st);
        return rc ? rc : join_product<T, ZNNI_ACT_NONE>(p.w, N, K, y.dw, st);
    }
    if (dbias && N > 0) {
        const znni_status rc = launch_sum_parts<T>(N, M > 0 ? slope_parts(M, N) : 0, SumOut<T>{{(T*)dbias}, {sums}}, 1, st);
        if (rc) return rc;
    }
    if (dx && M > 0 && K > 0) {
        End<T> d = end_of<T>(dx);
        d.parts = parts;
        const znni_status rc = launch_product<T, false, true, ZNNI_ACT_NONE>(M, K, N, side_of<T>(w, K), side_of<T>(&g, M), d, st);
        if (rc) return rc;
    }
    if (dw && N > 0 && K > 0) {
        End<T> d = end_of<T>(dw);
        d.parts = parts;
        const znni_status rc = launch_product<T, false, false, ZNNI_ACT_NONE>(N, K, M, side_of<T>(x, K), side_of<T>(&g, N), d, st);
        if (rc) return rc;
    }
    return ZNNI_OK;
}

static znni_status linear_shape(int type, int M, int N, int K)
{
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (M < 0 || N < 0 || K < 0 || M > ROWS_MOST || N > COLS_MOST || K > COLS_MOST) return ZNNI_ERR_SHAPE;
    return ZNNI_OK;
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_linear_workspace(int type, int M, int N, int K, size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    const znni_status rc = linear_shape(type, M, N, K);
    if (rc) return rc;
    *bytes = M > 0 && N > 0 ? up(product_plan(type, M, N, K, true).parts * sizeof(float)) : 0;
    return ZNNI_OK;
}

znni_status znni_linear(int type, int M, int N, int K, const znni_rows* x, const znni_rows* w, const void* bias, int act,
                        const znni_rows* residual, const znni_rows* z, const znni_rows* out, void* workspace, size_t workspace_bytes,
                        void* stream)
{
    if (!x || !w || !out) return ZNNI_ERR_NULL;
    if (act < ZNNI_ACT_NONE || act > ZNNI_ACT_SILU) return ZNNI_ERR_FLAGS;
    size_t need = 0;
    znni_status rc = znni_linear_workspace(type, M, N, K, &need);
    if (rc) return rc;
    if (M == 0 || N == 0) return ZNNI_OK;
    if ((rc = rows_fine(x, type, M, K, false)) || (rc = rows_fine(w, type, N, K, false)) || (rc = rows_fine(out, type, M, N, true))) return rc;
    if (residual && (rc = rows_fine(residual, type, M, N, false))) return rc;
    if (z && (rc = rows_fine(z, type, M, N, true))) return rc;
    if (need && !workspace) return ZNNI_ERR_NULL;
    if ((uintptr_t)bias % type_size(type) || (need && ((uintptr_t)workspace & 255u))) return ZNNI_ERR_ALIGN;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return forward<float>(M, N, K, x, w, bias, act, residual, z, out, workspace, st);
        case ZNNI_BF16: return forward<bf16>(M, N, K, x, w, bias, act, residual, z, out, workspace, st);
        default: return forward<f16>(M, N, K, x, w, bias, act, residual, z, out, workspace, st);
    }
}

znni_status znni_linear_backward_workspace(int type, int M, int N, int K, int act, unsigned wanted, size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    if (act < ZNNI_ACT_NONE || act > ZNNI_ACT_SILU || wanted & ~(ZNNI_LINEAR_DX | ZNNI_LINEAR_DW | ZNNI_LINEAR_DBIAS)) return ZNNI_ERR_FLAGS;
    const znni_status rc = linear_shape(type, M, N, K);
    if (rc) return rc;
    *bytes = backward_plan(type, M, N, K, act, wanted & ZNNI_LINEAR_DX, wanted & ZNNI_LINEAR_DW, wanted & ZNNI_LINEAR_DBIAS).all();
    return ZNNI_OK;
}

znni_status znni_linear_backward(int type, int M, int N, int K, const znni_rows* dout, const znni_rows* x, const znni_rows* w,
                                 const znni_rows* z, int act, const znni_rows* dx, const znni_rows* dw, void* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    if (!dout || (dw && !x) || (dx && !w)) return ZNNI_ERR_NULL;
    size_t need = 0;
    znni_status rc = znni_linear_backward_workspace(type, M, N, K, act, (dx ? ZNNI_LINEAR_DX : 0) | (dw ? ZNNI_LINEAR_DW : 0) | (dbias ? ZNNI_LINEAR_DBIAS : 0), &need);
    if (rc) return rc;
    if (act != ZNNI_ACT_NONE && !z) return ZNNI_ERR_NULL;
    if ((rc = rows_fine(dout, type, M, N, false))) return rc;
    if (act != ZNNI_ACT_NONE && (rc = rows_fine(z, type, M, N, false))) return rc;
    if (dw && ((rc = rows_fine(x, type, M, K, false)) || (rc = rows_fine(dw, type, N, K, true)))) return rc;
    if (dx && ((rc = rows_fine(w, type, N, K, false)) || (rc = rows_fine(dx, type, M, K, true)))) return rc;
    // (nothing wanted: the workspace has no place for dz either)
    if (!dx && !dw && !dbias) return ZNNI_OK;
    if (need && !workspace) return ZNNI_ERR_NULL;
    if ((uintptr_t)dbias % type_size(type) || (need && ((uintptr_t)workspace & 255u))) return ZNNI_ERR_ALIGN;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    if (act == ZNNI_ACT_NONE) z = nullptr;
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return backward<float>(type, M, N, K, dout, x, w, z, act, dx, dw, dbias, workspace, st);
        case ZNNI_BF16: return backward<bf16>(type, M, N, K, dout, x, w, z, act, dx, dw, dbias, workspace, st);
        default: return backward<f16>(type, M, N, K, dout, x, w, z, act, dx, dw, dbias, workspace, st);
    }
}

}  // extern "C"
