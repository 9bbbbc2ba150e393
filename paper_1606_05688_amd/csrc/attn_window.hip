// attn_window.hip -- attention with a sliding window and first tokens that stay visible, over sequences of any lengths.
#include "attn_common.h"

namespace znni {

struct AttnArgs {
    int Hq, Hk, D;
    const int* cu_q;
    const int* cu_k;
    Window w;
    float scale;
};

constexpr int AROW_THREADS = 256;

// One workgroup a row and head, as the formula has it: scores of 256 keys, running maximum and sum, weighted values.
template <typename T>
__global__ __launch_bounds__(AROW_THREADS) void k_attn_rows(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<T> out)
{
    __shared__ float qs[ATTN_DMAX], p[AROW_THREADS], red[AROW_THREADS / 64], sum2[ATTN_DMAX];
    const int b = blockIdx.z, h = blockIdx.y, i = blockIdx.x, t = threadIdx.x;
    const int nq = a.cu_q[b + 1] - a.cu_q[b], nk = a.cu_k[b + 1] - a.cu_k[b];
    if (i >= nq) return;
    const int hk = h / (a.Hq / a.Hk);
    const long long pos = (long long)nk - nq + i, k0 = a.cu_k[b];
    int lo, hi;
    window_of(pos, nk, a.w, &lo, &hi);
    const int first = min(min(a.w.sinks, lo), hi + 1), n = first + max(0, hi - lo + 1);
    const T* qr = q.row(a.cu_q[b] + (long long)i, h);
    for (int d = t; d < a.D; d += AROW_THREADS) qs[d] = (float)qr[d];
    float m = -INFINITY, l = 0.f, acc = 0.f;
    const int d = t & (ATTN_DMAX - 1), half = t / ATTN_DMAX;
    for (int j0 = 0; j0 < n; j0 += AROW_THREADS) {
        const int j = j0 + t, key = j < first ? j : lo + j - first;
        float s = -INFINITY;
        __syncthreads();
        if (j < n) {
            const T* kr = k.row(k0 + key, hk);
            s = 0.f;
            for (int e = 0; e < a.D; ++e) s += qs[e] * (float)kr[e];
            s *= a.scale;
        }
        float top = s;
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        if ((t & 63) == 0) red[t >> 6] = top;
        __syncthreads();
        float mn = m;
        for (int x = 0; x < AROW_THREADS / 64; ++x) mn = fmaxf(mn, red[x]);
        const float base = mn == -INFINITY ? 0.f : mn, old = expf(m - base);
        p[t] = j < n ? expf(s - base) : 0.f;
        m = mn;
        __syncthreads();
        l *= old;
        acc *= old;
        const int c = min(AROW_THREADS, n - j0);
        for (int x = 0; x < c; ++x) l += p[x];
        if (d < a.D)
            for (int x = half; x < c; x += AROW_THREADS / ATTN_DMAX) {
                const int y = j0 + x;
                acc += p[x] * (float)v.row(k0 + (y < first ? y : lo + y - first), hk)[d];
            }
    }
    __syncthreads();
    if (half) sum2[d] = acc;
    __syncthreads();
    if (!half && d < a.D) out.row(a.cu_q[b] + (long long)i, h)[d] = (T)(l == 0.f ? 0.f : (acc + sum2[d]) / l);
}

template <typename T>
static znni_status launch_attn(const AttnArgs& a, int B, int max_q, const znni_heads* q, const znni_heads* k, const znni_heads* v,
                               const znni_heads* out, hipStream_t st)
{
    k_attn_rows<T><<<dim3((unsigned)max_q, (unsigned)a.Hq, (unsigned)B), dim3(AROW_THREADS), 0, st>>>(
        a, heads_of<const T>(q), heads_of<const T>(k), heads_of<const T>(v), heads_of<T>(out));
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

static znni_status attn_shape(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks)
{
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (B < 0 || B > 65535 || max_q < 0 || max_k < 0 || left < 0 || right < 0 || sinks < 0) return ZNNI_ERR_SHAPE;
    return heads_shape(Hq, Hk, D);
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_attn_window_workspace(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks,
                                       size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    const znni_status rc = attn_shape(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
    if (rc) return rc;
    *bytes = 0;
    return ZNNI_OK;
}

znni_status znni_attn_window(int type, int B, int Hq, int Hk, int D, const znni_heads* q, const znni_heads* k, const znni_heads* v,
                             const int* cu_q, const int* cu_k, int max_q, int max_k, int left, int right, int sinks, float scale,
                             const znni_heads* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !k || !v || !out) return ZNNI_ERR_NULL;
    size_t need = 0;
    const znni_status rc = znni_attn_window_workspace(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks, &need);
    if (rc) return rc;
    if (B == 0 || max_q == 0) return ZNNI_OK;
    if (!q->data || !out->data || (max_k > 0 && (!k->data || !v->data)) || !cu_q || !cu_k || (need && !workspace)) return ZNNI_ERR_NULL;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k) & 3u || (need && ((uintptr_t)workspace & 255u))) return ZNNI_ERR_ALIGN;
    for (const znni_heads* h : {q, k, v, out})
        if (!heads_aligned(h, type)) return ZNNI_ERR_ALIGN;
    const AttnArgs a = {Hq, Hk, D, cu_q, cu_k, {left, right, sinks}, scale};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_attn<float>(a, B, max_q, q, k, v, out, st);
        case ZNNI_BF16: return launch_attn<bf16>(a, B, max_q, q, k, v, out, st);
        default: return launch_attn<f16>(a, B, max_q, q, k, v, out, st);
    }
}

}  // extern "C"
