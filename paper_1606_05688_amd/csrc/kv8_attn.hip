// kv8_attn.hip -- attention of the last tokens of sequences over the 8-bit cache.
#include "kv8.h"

namespace znni {

struct Kv8Args {
    int Lq, Hq, Hk, D, pages, width;
    const unsigned char* kcodes;
    const unsigned char* vcodes;
    const float* scales;
    const int* table;
    const int* lens;
    Window w;
    float scale;
};

constexpr int KROW_THREADS = 256;

__device__ inline float value_of(unsigned char code) { return __builtin_amdgcn_cvt_f32_fp8(code, 0); }

// One workgroup a row and head, as the formula has it.
template <typename T>
__global__ __launch_bounds__(KROW_THREADS) void k_kv8_rows(Kv8Args a, Heads<const T> q, Heads<T> out)
{
    __shared__ float qs[ATTN_DMAX], p[KROW_THREADS], red[KROW_THREADS / 64], sum2[ATTN_DMAX];
    const int b = blockIdx.z, h = blockIdx.y, i = blockIdx.x, t = threadIdx.x;
    const int nk = (int)min((long long)a.lens[b], (long long)a.width * PAGE);
    const int hk = h / (a.Hq / a.Hk);
    const long long pos = (long long)nk - a.Lq + i;
    int lo, hi;
    window_of(pos, nk, a.w, &lo, &hi);
    const int first = min(min(a.w.sinks, lo), hi + 1), n = first + max(0, hi - lo + 1);
    const T* qr = q.row((long long)b * a.Lq + i, h);
    for (int d = t; d < a.D; d += KROW_THREADS) qs[d] = (float)qr[d];
    float m = -INFINITY, l = 0.f, acc = 0.f;
    const int d = t & (ATTN_DMAX - 1), half = t / ATTN_DMAX;
    for (int j0 = 0; j0 < n; j0 += KROW_THREADS) {
        const int j = j0 + t, key = j < first ? j : lo + j - first;
        float s = -INFINITY;
        __syncthreads();
        const int page = j < n ? a.table[(long long)b * a.width + key / PAGE] : -1;
        const bool there = page >= 0 && page < a.pages;
        const long long at = (long long)page * a.Hk + hk;
        if (there) {
            const unsigned char* kr = a.kcodes + (at * PAGE + key % PAGE) * a.D;
            s = 0.f;
            for (int e = 0; e < a.D; ++e) s += qs[e] * value_of(kr[e]);
            s *= a.scale * a.scales[at * 2];
        }
        float top = s;
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        if ((t & 63) == 0) red[t >> 6] = top;
        __syncthreads();
        float mn = m;
        for (int x = 0; x < KROW_THREADS / 64; ++x) mn = fmaxf(mn, red[x]);
        const float base = mn == -INFINITY ? 0.f : mn, old = expf(m - base);
        p[t] = there ? expf(s - base) : 0.f;
        m = mn;
        __syncthreads();
        l *= old;
        acc *= old;
        const int c = min(KROW_THREADS, n - j0);
        for (int x = 0; x < c; ++x) l += p[x];
        if (d < a.D)
            for (int x = half; x < c; x += KROW_THREADS / ATTN_DMAX) {
                const int y = j0 + x, kv = y < first ? y : lo + y - first, pg = a.table[(long long)b * a.width + kv / PAGE];
                if (pg < 0 || pg >= a.pages) continue;
                const long long o = (long long)pg * a.Hk + hk;
                acc += p[x] * (value_of(a.vcodes[(o * a.D + d) * PAGE + kv % PAGE]) * a.scales[o * 2 + 1]);
            }
    }
    __syncthreads();
    if (half) sum2[d] = acc;
    __syncthreads();
    if (!half && d < a.D) out.row((long long)b * a.Lq + i, h)[d] = (T)(l == 0.f ? 0.f : (acc + sum2[d]) / l);
}

template <typename T>
static znni_status launch_kv8(const Kv8Args& a, int B, const znni_heads* q, const znni_heads* out, hipStream_t st)
{
    k_kv8_rows<T><<<dim3((unsigned)a.Lq, (unsigned)a.Hq, (unsigned)B), dim3(KROW_THREADS), 0, st>>>(a, heads_of<const T>(q), heads_of<T>(out));
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
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
    *bytes = 0;
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
    const Kv8Args a = {Lq, Hq, Hk, D, pages, width, kcodes, vcodes, scales, table, lens, {left, 0, sinks}, scale};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_kv8<float>(a, B, q, out, st);
        case ZNNI_BF16: return launch_kv8<bf16>(a, B, q, out, st);
        default: return launch_kv8<f16>(a, B, q, out, st);
    }
}

}  // extern "C"
