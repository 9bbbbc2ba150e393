// block_norm.hip -- norms where a block ends and the next one begins, with the block's gate and scale, and their gradients.
//
//   h = x + scale * gate * post * n(y),   z = pre * n(h),   n(a) = a r,  r = 1 / sqrt(mean a^2 + eps)   (centred: of a - mean a)
//   gradients: dx = dh + n'(h)[pre dz],   n'(a)[g] = r (g - n(a) mean(g n(a)))   (centred: less its mean);
//   dgate = scale dx post n(y),   dy = n'(y)[scale dx gate post],   dpost = sum over tokens of scale dx gate n(y),   dpre = of dz n(h)
//
// Bound by memory: every tensor is read or written once.  Rows stay in registers, 8 to 32 elements a lane, one to sixteen waves a row (but for gradients past
// 8192 channels, whose rows, weights and sums are more than sixteen waves hold: 400 to 464 bytes of scratch a lane, 4096 x 16384 bf16 824 us, 1 TB/s).
// bf16, 32768 x 2048, a gate for each token: 117 us, 5.7 TB/s (a large copy reaches 5.2 to 6.2 by card).  Gradients, one gate: 183 to 194 us, 4.2 to 4.4
// TB/s, and 6 for the sums over tokens: a row over four waves, four workgroups a compute unit, three meetings a row; 32 elements a lane and a wave a
// row leave two waves a SIMD and took 285; the next row's reads ahead of this one's work cost a workgroup and took 209.
#include <initializer_list>
#include <type_traits>

#include "rows_common.h"

namespace znni {

struct NormArgs {
    int T, C, per;                       // per: rows of a workgroup
    float scale, eps;
    bool post, pre, centred;             // whether y and h are normed, whether means are taken off
    bool shared;                         // one gate for all tokens
};

template <typename T>
struct Rows {
    T* p;
    long long row;
};

template <typename T>
static Rows<T> rows_of(const znni_rows* r)
{
    return r ? Rows<T>{(T*)r->data, r->row} : Rows<T>{nullptr, 0};
}

// A row over the lanes of W waves: E elements a lane in vectors of VEC.
template <typename T, int VEC, int E, int W>
struct Row {
    static constexpr int LANES = 64 * W, NV = E / VEC;
    typedef T V __attribute__((ext_vector_type(VEC)));
    __device__ static int column(int lane, int v) { return (v * LANES + lane) * VEC; }
    __device__ static void load(V (&y)[NV], const T* p, int lane, int C)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = column(lane, v);
            y[v] = Loose<T, VEC>::load(p + c, C - c);
        }
    }
    __device__ static void clear(V (&y)[NV])
    {
#pragma unroll
        for (int i = 0; i < E; ++i) y[i / VEC][i % VEC] = (T)0.f;
    }
    // Sums of a pair over the row.  Waves meet once: a sum's place in LDS is written again two sums later.
    struct Sums {
        float2 (*place)[W];
        int turn;
        __device__ float2 operator()(float2 x)
        {
#pragma unroll
            for (int o = 32; o; o >>= 1) x.x += __shfl_xor(x.x, o), x.y += __shfl_xor(x.y, o);
            if constexpr (W > 1) {
                turn ^= 1;
                if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6] = x;
                __syncthreads();
                x = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < W; ++i) x.x += place[turn][i].x, x.y += place[turn][i].y;
            }
            return x;
        }
    };
};

// Means (or 0) and factors of two rows, `first` and `second` (as far as they are normed); lanes past their end hold zeros.
template <typename R, int E, int VEC, typename F, typename G>
__device__ inline void moments(F first, G second, const NormArgs& a, bool one, bool two, int lane, typename R::Sums& sum, float2* mean, float2* r)
{
    float2 m = {0.f, 0.f}, s = {0.f, 0.f};
    if (a.centred) {
#pragma unroll
        for (int i = 0; i < E; ++i) s.x += first(i), s.y += second(i);
        s = sum(s);
        m = make_float2(one ? s.x / a.C : 0.f, two ? s.y / a.C : 0.f);
        s = make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const bool there = R::column(lane, i / VEC) + i % VEC < a.C;
        const float x = there ? first(i) - m.x : 0.f, y = there ? second(i) - m.y : 0.f;
        s.x = fmaf(x, x, s.x);
        s.y = fmaf(y, y, s.y);
    }
    s = sum(s);
    *mean = m;
    *r = make_float2(one ? 1.f / sqrtf(s.x / a.C + a.eps) : 1.f, two ? 1.f / sqrtf(s.y / a.C + a.eps) : 1.f);
}

template <typename T, int VEC, int E, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(NormArgs a, Rows<const T> x, Rows<const T> y, Rows<const T> gate, const T* post, const T* pre,
                                                               Rows<T> h, Rows<T> z)
{
    using R = Row<T, VEC, E, W>;
    typedef typename R::V V;
    constexpr int NV = R::NV;
    __shared__ float2 place[2][W];
    typename R::Sums sum = {place, 0};
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const long long t = W == 1 ? group_id() * 4 + (threadIdx.x >> 6) : group_id();
    if (t >= a.T) return;
    V xv[NV];
    R::load(xv, x.p + t * x.row, lane, a.C);
    float s[E];
#pragma unroll
    for (int i = 0; i < E; ++i) s[i] = (float)xv[i / VEC][i % VEC];
    const auto none = [](int) { return 0.f; };
    float2 mean = {0.f, 0.f}, r = {1.f, 1.f};
    if (y.p) {
        V yv[NV], w[NV], g[NV];
        R::load(yv, y.p + t * y.row, lane, a.C);
        if (gate.p) R::load(g, gate.p + t * gate.row, lane, a.C);
        if (post) R::load(w, post, lane, a.C);
        if (a.post) moments<R, E, VEC>([&](int i) { return (float)yv[i / VEC][i % VEC]; }, none, a, true, false, lane, sum, &mean, &r);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float u = ((float)yv[i / VEC][i % VEC] - mean.x) * r.x;
            if (post) u *= (float)w[i / VEC][i % VEC];
            if (gate.p) u *= (float)g[i / VEC][i % VEC];
            s[i] += a.scale * u;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            V o;
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = (T)s[v * VEC + e];
            const int c = R::column(lane, v);
            if (c < a.C) Loose<T, VEC>::store(h.p + t * h.row + c, o, a.C - c);
            // (past the row's end: whatever a mean taken off has left)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[v * VEC + e] = c + e < a.C ? s[v * VEC + e] : 0.f;
        }
    }
    if (!a.pre) return;
    V w[NV];
    if (pre) R::load(w, pre, lane, a.C);
    moments<R, E, VEC>([&](int i) { return s[i]; }, none, a, true, false, lane, sum, &mean, &r);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (R::column(lane, v) >= a.C) continue;
        V o;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float n = (s[v * VEC + e] - mean.x) * r.x;
            if (pre) n *= (float)w[v][e];
            o[e] = (T)n;
        }
        Loose<T, VEC>::store(z.p + t * z.row + R::column(lane, v), o, a.C - R::column(lane, v));
    }
}

// Where sums over tokens go: [workgroup][C] each, or NULL.
struct NormSums {
    float *gate, *post, *pre;
};

template <typename T, int VEC, int E, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm_back(NormArgs a, Rows<const T> dh, Rows<const T> dz, Rows<const T> h, Rows<const T> y,
                                                                    Rows<const T> gate, const T* post, const T* pre, Rows<T> dx, Rows<T> dy,
                                                                    Rows<T> dgate, NormSums sums)
{
    using R = Row<T, VEC, E, W>;
    typedef typename R::V V;
    constexpr int NV = R::NV, AT_ONCE = W == 1 ? 4 : 1;
    __shared__ float2 place[2][W];
    __shared__ float joined[W == 1 ? 4 * 64 * E : 1];
    typename R::Sums sum = {place, 0};
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, mine = W == 1 ? threadIdx.x >> 6 : 0;
    const long long t0 = group_id() * a.per, t1 = min((long long)a.T, t0 + a.per);
    float sg[E], sp[E], sq[E];
#pragma unroll
    for (int i = 0; i < E; ++i) sg[i] = sp[i] = sq[i] = 0.f;
    // What a call does not have takes part as what changes nothing (ones, and zeros for means and sums): every element goes the same way.
    V wq[NV], wp[NV];
    auto weights = [&](V (&w)[NV], const T* p) {
        if (p) R::load(w, p, lane, a.C);
        else
#pragma unroll
            for (int i = 0; i < E; ++i) w[i / VEC][i % VEC] = (T)(R::column(lane, i / VEC) + i % VEC < a.C ? 1.f : 0.f);
    };
    weights(wq, pre);
    weights(wp, post);
    V one[NV];                                         // a gate that all tokens share, or none
    if (!gate.p || a.shared) weights(one, gate.p);
    const bool block = y.p || dy.p;
    for (long long t = t0 + mine; t < t1; t += AT_ONCE) {
        // all of the row's reads first
        V hv[NV], zv[NV], xv[NV], yv[NV], gv[NV];
        if (a.pre) R::load(hv, h.p + t * h.row, lane, a.C), R::load(zv, dz.p + t * dz.row, lane, a.C);
        else R::clear(hv), R::clear(zv);
        if (dh.p) R::load(xv, dh.p + t * dh.row, lane, a.C);
        else R::clear(xv);
        if (y.p) R::load(yv, y.p + t * y.row, lane, a.C);
        else R::clear(yv);
        if (gate.p && !a.shared) R::load(gv, gate.p + t * gate.row, lane, a.C);
        else
#pragma unroll
            for (int v = 0; v < NV; ++v) gv[v] = one[v];
        auto of = [](const V (&x)[NV], int i) { return (float)x[i / VEC][i % VEC]; };
        auto put = [&](const Rows<T>& to, auto at) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (R::column(lane, v) >= a.C) continue;
                V o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = (T)at(v * VEC + e);
                Loose<T, VEC>::store(to.p + t * to.row + R::column(lane, v), o, a.C - R::column(lane, v));
            }
        };
        float2 mean = {0.f, 0.f}, r = {1.f, 1.f};
        if (a.pre || a.post) moments<R, E, VEC>([&](int i) { return of(hv, i); }, [&](int i) { return of(yv, i); }, a, a.pre, a.post, lane, sum, &mean, &r);
        const float hm = mean.x, hr = r.x, ym = mean.y, yr = r.y;
        float d[E];
        float2 over = {0.f, 0.f};                          // of the gradient times the normed row, of the gradient
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float n = (of(hv, i) - hm) * hr, z = of(zv, i);
            sq[i] = fmaf(z, n, sq[i]);
            d[i] = z * of(wq, i);
            over.x = fmaf(d[i], n, over.x);
            over.y += d[i];
        }
        if (a.pre) {
            over = sum(over);
            over = make_float2(over.x / a.C, a.centred ? over.y / a.C : 0.f);
        } else {
            over = make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] = fmaf(hr, d[i] - (of(hv, i) - hm) * hr * over.x - over.y, of(xv, i));
        if (dx.p) put(dx, [&](int i) { return d[i]; });
        if (!block) continue;
        auto normed = [&](int i) { return (of(yv, i) - ym) * yr; };
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] *= a.scale;
        if (dgate.p) put(dgate, [&](int i) { return d[i] * (normed(i) * of(wp, i)); });
        over = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float n = normed(i);
            sg[i] = fmaf(d[i], n * of(wp, i), sg[i]);
            d[i] *= of(gv, i);
            sp[i] = fmaf(d[i], n, sp[i]);
            d[i] *= of(wp, i);
            over.x = fmaf(d[i], n, over.x);
            over.y += d[i];
        }
        if (a.post) {
            over = sum(over);
            over = make_float2(over.x / a.C, a.centred ? over.y / a.C : 0.f);
#pragma unroll
            for (int i = 0; i < E; ++i) d[i] = yr * (d[i] - normed(i) * over.x - over.y);
        }
        // (without a norm y has no part in its gradient: an infinity in it would make NaN of a product with zero)
        if (dy.p) put(dy, [&](int i) { return d[i]; });
    }
    auto write = [&](float* to, const float (&s)[E]) {
        if (!to) return;
        to += group_id() * a.C;
        if constexpr (W == 1) {
            // the four waves' sums, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < E; ++i) joined[(mine * E + i) * 64 + lane] = s[i];
            __syncthreads();
            for (int i = mine; i < E; i += 4) {
                const int c = R::column(lane, i / VEC) + i % VEC;
                if (c < a.C) to[c] = (joined[i * 64 + lane] + joined[(E + i) * 64 + lane]) + (joined[(2 * E + i) * 64 + lane] + joined[(3 * E + i) * 64 + lane]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int c = R::column(lane, i / VEC) + i % VEC;
                if (c < a.C) to[c] = s[i];
            }
        }
    };
    write(sums.gate, sg);
    write(sums.post, sp);
    write(sums.pre, sq);
}

constexpr int NORM_MOST = 16384;          // channels
constexpr int NORM_GROUPS = 1024;         // workgroups that share the rows, where sums over tokens are wanted

// Elements a lane and waves a row.
struct NormShape {
    int E, W;
};
static NormShape norm_shape(int T, int C)
{
    if (C <= 512) return {8, 1};
    if (C <= 2048) return T <= 1024 ? NormShape{8, 4} : NormShape{32, 1};
    return {32, C <= 4096 ? 2 : C <= 8192 ? 4 : 8};
}
// Gradients hold five rows and three sums.
static NormShape norm_back_shape(int C)
{
    return C <= 512 ? NormShape{8, 1} : C <= 2048 ? NormShape{8, 4} : C <= 4096 ? NormShape{8, 8} : NormShape{16, C <= 8192 ? 8 : 16};
}

// Rows of a workgroup: with sums over tokens, all those that make NORM_GROUPS workgroups.
static int norm_rows(int T, int W, bool sums)
{
    const int once = W == 1 ? 4 : 1;
    if (!sums) return once;
    const long long n = ((long long)T + NORM_GROUPS - 1) / NORM_GROUPS;
    return (int)((n + once - 1) / once * once);
}

// Workgroups that leave sums over tokens, at most: of more rows never fewer, so that a workspace does for all smaller calls.
static long long norm_parts(int T, int C)
{
    const int once = norm_back_shape(C).W == 1 ? 4 : 1;
    const long long n = ((long long)T + once - 1) / once;
    return n < NORM_GROUPS ? n : NORM_GROUPS;
}
static size_t norm_sums(int T, int C) { return up((size_t)norm_parts(T, C) * C * sizeof(float)); }

template <typename T, typename F>
static znni_status with_row(NormShape s, F f)
{
    constexpr int V = 16 / sizeof(T);
    if (s.E == 8) s.W == 1 ? f(Row<T, V, 8, 1>()) : f(Row<T, V, 8, 4>());
    else s.W == 1 ? f(Row<T, V, 32, 1>()) : s.W == 2 ? f(Row<T, V, 32, 2>()) : s.W == 4 ? f(Row<T, V, 32, 4>()) : f(Row<T, V, 32, 8>());
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

template <typename T, typename F>
static znni_status with_back_row(NormShape s, F f)
{
    constexpr int V = 16 / sizeof(T);
    if (s.E == 8) s.W == 1 ? f(Row<T, V, 8, 1>()) : s.W == 4 ? f(Row<T, V, 8, 4>()) : f(Row<T, V, 8, 8>());
    else s.W == 8 ? f(Row<T, V, 16, 8>()) : f(Row<T, V, 16, 16>());
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

template <typename T, int VEC, int E, int W, typename... A>
static void launch_norm(Row<T, VEC, E, W>, long long groups, hipStream_t st, A... args)
{
    constexpr unsigned THREADS = W == 1 ? 256 : 64 * W;
    k_norm<T, VEC, E, W><<<launch_of(groups, THREADS), dim3(THREADS), 0, st>>>(args...);
}

template <typename T, int VEC, int E, int W, typename... A>
static void launch_norm_back(Row<T, VEC, E, W>, long long groups, hipStream_t st, A... args)
{
    constexpr unsigned THREADS = W == 1 ? 256 : 64 * W;
    k_norm_back<T, VEC, E, W><<<launch_of(groups, THREADS), dim3(THREADS), 0, st>>>(args...);
}

template <typename T>
static znni_status norm_forward(NormArgs a, const znni_rows* x, const znni_rows* y, const znni_rows* gate, const void* post, const void* pre,
                                const znni_rows* h, const znni_rows* z, hipStream_t st)
{
    const long long groups = ((long long)a.T + a.per - 1) / a.per;
    Rows<const T> g = rows_of<const T>(gate);
    if (a.shared) g.row = 0;
    return with_row<T>(norm_shape(a.T, a.C), [&](auto row) {
        launch_norm(row, groups, st, a, rows_of<const T>(x), rows_of<const T>(y), g, (const T*)post, (const T*)pre, rows_of<T>(h), rows_of<T>(z));
        return 0;
    });
}

template <typename T>
static znni_status norm_backward(NormArgs a, const znni_rows* dh, const znni_rows* dz, const znni_rows* h, const znni_rows* y, const znni_rows* gate,
                                 const void* post, const void* pre, const znni_rows* dx, const znni_rows* dy, const znni_rows* dgate, void* dpost,
                                 void* dpre, float* workspace, hipStream_t st)
{
    Rows<const T> g = rows_of<const T>(gate);
    if (a.shared) g.row = 0;
    const bool summed = a.shared && dgate;
    const long long groups = a.T ? ((long long)a.T + a.per - 1) / a.per : 0;
    const size_t step = norm_sums(a.T, a.C) / sizeof(float);
    NormSums sums = {};
    SumOut<T> o = {};
    int n = 0;
    auto wants = [&](bool wanted, void* to) -> float* {
        if (!wanted) return nullptr;
        float* from = workspace + n * step;
        o.to[n] = (T*)to;
        o.from[n++] = from;
        return from;
    };
    sums.gate = wants(summed, summed ? dgate->data : nullptr);
    sums.post = wants(dpost, dpost);
    sums.pre = wants(dpre, dpre);
    if (a.T > 0) {
        const Rows<T> dg = summed ? Rows<T>{nullptr, 0} : rows_of<T>(dgate);
        const znni_status rc = with_back_row<T>(norm_back_shape(a.C), [&](auto row) {
            launch_norm_back(row, groups, st, a, rows_of<const T>(dh), rows_of<const T>(dz), rows_of<const T>(h), rows_of<const T>(y), g,
                             (const T*)post, (const T*)pre, rows_of<T>(dx), rows_of<T>(dy), dg, sums);
            return 0;
        });
        if (rc) return rc;
    }
    return n ? launch_sum_parts<T>(a.C, (int)groups, o, n, st) : ZNNI_OK;
}

static znni_status norm_shape_fine(int type, int T, int C, unsigned flags)
{
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (flags & ~(ZNNI_NORM_POST | ZNNI_NORM_PRE | ZNNI_NORM_CENTRED | ZNNI_NORM_GATE_SHARED)) return ZNNI_ERR_FLAGS;
    if (T < 0 || C < 1 || T > ROWS_MOST) return ZNNI_ERR_SHAPE;
    return C > NORM_MOST ? ZNNI_ERR_UNSUPPORTED_SIZE : ZNNI_OK;
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_block_norm(int type, int T, int C, const znni_rows* x, const znni_rows* y, const znni_rows* gate, const void* post, const void* pre,
                            float scale, float eps, unsigned flags, const znni_rows* h, const znni_rows* z, void* stream)
{
    znni_status rc = norm_shape_fine(type, T, C, flags);
    if (rc) return rc;
    const bool has_pre = flags & ZNNI_NORM_PRE, has_post = flags & ZNNI_NORM_POST, shared = flags & ZNNI_NORM_GATE_SHARED;
    if (!x || !y != !h || (has_pre && !z)) return ZNNI_ERR_NULL;
    // what a call does not use has no place in it
    if ((!y && (gate || has_post)) || (post && !has_post) || ((pre || z) && !has_pre) || (shared && !gate) || (!y && !has_pre)) return ZNNI_ERR_FLAGS;
    if (T == 0) return ZNNI_OK;
    if ((rc = rows_fine(x, type, T, C, false)) || (has_pre && (rc = rows_fine(z, type, T, C, true)))) return rc;
    if (y && ((rc = rows_fine(y, type, T, C, false)) || (rc = rows_fine(h, type, T, C, true)))) return rc;
    if (gate && (rc = rows_fine(gate, type, shared ? 1 : T, C, false))) return rc;
    if (((uintptr_t)post | (uintptr_t)pre) % type_size(type)) return ZNNI_ERR_ALIGN;
    const NormArgs a = {T, C, norm_rows(T, norm_shape(T, C).W, false), scale, eps, has_post, has_pre, (flags & ZNNI_NORM_CENTRED) != 0, shared};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return norm_forward<float>(a, x, y, gate, post, pre, h, z, st);
        case ZNNI_BF16: return norm_forward<bf16>(a, x, y, gate, post, pre, h, z, st);
        default: return norm_forward<f16>(a, x, y, gate, post, pre, h, z, st);
    }
}

znni_status znni_block_norm_backward_workspace(int type, int T, int C, unsigned flags, size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    const znni_status rc = norm_shape_fine(type, T, C, flags);
    if (rc) return rc;
    *bytes = 3 * norm_sums(T, C);
    return ZNNI_OK;
}

znni_status znni_block_norm_backward(int type, int T, int C, const znni_rows* dh, const znni_rows* dz, const znni_rows* h, const znni_rows* y,
                                     const znni_rows* gate, const void* post, const void* pre, float scale, float eps, unsigned flags,
                                     const znni_rows* dx, const znni_rows* dy, const znni_rows* dgate, void* dpost, void* dpre, void* workspace,
                                     size_t workspace_bytes, void* stream)
{
    size_t need = 0;
    znni_status rc = znni_block_norm_backward_workspace(type, T, C, flags, &need);
    if (rc) return rc;
    const bool has_pre = flags & ZNNI_NORM_PRE, has_post = flags & ZNNI_NORM_POST, shared = flags & ZNNI_NORM_GATE_SHARED;
    if ((has_pre && (!h || !dz)) || (!has_pre && !dh)) return ZNNI_ERR_NULL;
    if ((has_post || dgate || dpost) && !y) return ZNNI_ERR_NULL;
    if (dgate && !gate) return ZNNI_ERR_NULL;
    if ((post && !has_post) || (dpost && !has_post) || ((pre || dz || dpre) && !has_pre) || (shared && !gate)) return ZNNI_ERR_FLAGS;
    const bool summed = (shared && dgate) || dpost || dpre;
    if ((rc = dh ? rows_fine(dh, type, T, C, false) : ZNNI_OK)) return rc;
    if (has_pre && ((rc = rows_fine(dz, type, T, C, false)) || (rc = rows_fine(h, type, T, C, false)))) return rc;
    if (y && (rc = rows_fine(y, type, T, C, false))) return rc;
    if (gate && (rc = rows_fine(gate, type, shared ? 1 : T, C, false))) return rc;
    for (const znni_rows* o : {dx, dy})
        if (o && (rc = rows_fine(o, type, T, C, true))) return rc;
    if (dgate && (rc = rows_fine(dgate, type, shared ? 1 : T, C, true))) return rc;
    if (((uintptr_t)post | (uintptr_t)pre | (uintptr_t)dpost | (uintptr_t)dpre) % type_size(type)) return ZNNI_ERR_ALIGN;
    if (summed && need) {
        if (!workspace) return ZNNI_ERR_NULL;
        if ((uintptr_t)workspace & 255u) return ZNNI_ERR_ALIGN;
        if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    }
    const NormArgs a = {T, C, norm_rows(T, norm_back_shape(C).W, summed), scale, eps, has_post, has_pre, (flags & ZNNI_NORM_CENTRED) != 0, shared};
    float* const ws = (float*)workspace;
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return norm_backward<float>(a, dh, dz, h, y, gate, post, pre, dx, dy, dgate, dpost, dpre, ws, st);
        case ZNNI_BF16: return norm_backward<bf16>(a, dh, dz, h, y, gate, post, pre, dx, dy, dgate, dpost, dpre, ws, st);
        default: return norm_backward<f16>(a, dh, dz, h, y, gate, post, pre, dx, dy, dgate, dpost, dpre, ws, st);
    }
}

}  // extern "C"
