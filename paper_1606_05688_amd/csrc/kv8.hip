// kv8.hip -- filling the 8-bit cache of keys and values.
//
// A workgroup has one page and head.  A thread has four tokens of eight elements, of keys and of values, all loaded at once;
// the largest magnitudes meet in LDS, then codes go out: keys as they come (lanes along the head), values with the tokens innermost
// (lanes along the tokens: four codes of an element are a word, sixteen lanes a row of the page).  Bound by memory for prompts, by the
// chain of dependent reads (start, page, tokens and scale) for single tokens.  bf16, 2 sequences of 16384 tokens, heads 8 x 128, 201 MB:
// 37 us, 5.4 TB/s; one token for each of 64 sequences: 7.7 us.
#include "kv8.h"

namespace znni {

struct AppendArgs {
    int Hk, D, pages, width;
    const int* cu;
    const int* start;
    const int* table;
    unsigned char* kcodes;
    unsigned char* vcodes;
    float* scales;
};

constexpr int APPEND_THREADS = 256;
constexpr int GROUPS = PAGE / 4;         // of four tokens
static_assert(GROUPS * ATTN_DMAX / 8 <= APPEND_THREADS, "a unit for every thread");

// The least E >= -126 for which a <= 448 * 2^E = 1.75 * 2^(E + 8), a finite and not negative.
__device__ inline int exponent_of(float a)
{
    const int e = (int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 127 - 8;      // carries if the mantissa is over .75
    return e < -126 ? -126 : e;
}

__device__ inline float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }     // -126 .. 127

__device__ inline float e4m3_range(float y) { return fabsf(y) > 448.f ? copysignf(448.f, y) : y; }      // NaN stays NaN

// Four values, already scaled, as codes: nearest, ties to even.
__device__ inline unsigned codes_of(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(a), e4m3_range(b), 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(c), e4m3_range(d), r, true);
}

// Four codes times a power of two, rounded again.
__device__ inline unsigned rescaled(unsigned x, float by)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    return codes_of(a[0] * by, a[1] * by, b[0] * by, b[1] * by);
}

__device__ inline float largest(float a, float x)
{
    const float m = fabsf(x);
    return m <= 3.402823466e38f ? fmaxf(a, m) : a;       // infinities and NaN do not count
}

// Eight elements as they lie in memory.
template <typename T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
    V v[sizeof(T) / 2];
    __device__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = ((const V*)p)[i];
    }
    __device__ float at(int e) const { return (float)v[e * sizeof(T) / 16][e % (16 / (int)sizeof(T))]; }
};

// The scale of the page after these tokens; *grown is what older codes are multiplied by.
__device__ inline float new_scale(float top, float was, bool has_old, float* grown)
{
    int E = exponent_of(top);
    *grown = 1.f;
    if (has_old) {
        const int before = (int)(__float_as_uint(was) >> 23 & 255) - 127;
        if (before >= E) E = before;
        else *grown = power_of_two(before - E > -126 ? before - E : -126);
    }
    return power_of_two(E);
}

__device__ inline float inverse(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }     // of 2^-126 .. 2^120

template <typename T>
__global__ __launch_bounds__(APPEND_THREADS) void k_append(AppendArgs a, Heads<const T> k, Heads<const T> v)
{
    __shared__ float2 red[APPEND_THREADS / 64];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int c0 = a.cu[b], n = a.cu[b + 1] - c0, start = a.start[b];
    const long long index = (long long)start / PAGE + blockIdx.x, base = index * PAGE;
    const int s0 = (int)(start > base ? start - base : 0);                       // slots s0 .. s1 are new, those before s0 old
    const int s1 = (int)min((long long)PAGE, (long long)start + n - base);
    if (s0 >= s1 || start < 0 || index >= a.width) return;
    const int per = a.D / 8;
    const bool has = t < GROUPS * per;
    const int kd = t % per * 8, ks = t / per * 4, vd = t / GROUPS * 8, vs = t % GROUPS * 4;      // first element and slot of the units
    const long long token = c0 + base - start;
    // (slots of a unit that are not new: some new one, which counts once more and is not written; no branch for each, so that
    // all loads go out at once)
    Eight<T> x[4] = {}, y[4] = {};
    float2 top = {0.f, 0.f};
    if (has && ks < s1 && ks + 4 > s0)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(k.row(token + min(max(ks + i, s0), s1 - 1), h) + kd);
    if (has && vs < s1 && vs + 4 > s0)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i].load(v.row(token + min(max(vs + i, s0), s1 - 1), h) + vd);
    const int page = a.table[(long long)b * a.width + index];
    if (page < 0 || page >= a.pages) return;
    const long long at = (long long)page * a.Hk + h;
    float2* scale = (float2*)a.scales + at;
    const float2 was = *scale;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top.x = largest(top.x, x[i].at(e));
            top.y = largest(top.y, y[i].at(e));
        }
    for (int o = 32; o; o >>= 1) {
        top.x = fmaxf(top.x, __shfl_xor(top.x, o));
        top.y = fmaxf(top.y, __shfl_xor(top.y, o));
    }
    if ((t & 63) == 0) red[t >> 6] = top;
    __syncthreads();                          // (every thread has read the old scale, too)
#pragma unroll
    for (int w = 0; w < APPEND_THREADS / 64; ++w) {
        top.x = fmaxf(top.x, red[w].x);
        top.y = fmaxf(top.y, red[w].y);
    }
    float kg, vg;
    const float kscale = new_scale(top.x, was.x, s0 > 0, &kg), vscale = new_scale(top.y, was.y, s0 > 0, &vg);
    if (t == 0) *scale = make_float2(kscale, vscale);
    if (!has) return;
    const float kby = inverse(kscale), vby = inverse(vscale);
    unsigned char* kc = a.kcodes + at * PAGE * a.D;
    unsigned char* vc = a.vcodes + at * PAGE * a.D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint2* to = (uint2*)(kc + (ks + i) * a.D + kd);
        const Eight<T>& f = x[i];
        if (ks + i >= s1) continue;
        if (ks + i >= s0)
            *to = make_uint2(codes_of(f.at(0) * kby, f.at(1) * kby, f.at(2) * kby, f.at(3) * kby),
                             codes_of(f.at(4) * kby, f.at(5) * kby, f.at(6) * kby, f.at(7) * kby));
        else if (kg != 1.f) *to = make_uint2(rescaled(to->x, kg), rescaled(to->y, kg));
    }
    // values: slots vs .. vs + 3 of eight elements
    if (vs >= s1 || (vs + 4 <= s0 && vg == 1.f)) return;
    unsigned fresh = 0;                       // bytes that are new, and that are older tokens'
    unsigned older = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (vs + i >= s0 && vs + i < s1) fresh |= 255u << (8 * i);
        if (vs + i < s0) older |= 255u << (8 * i);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        unsigned* to = (unsigned*)(vc + (vd + e) * PAGE + vs);
        unsigned w = codes_of(y[0].at(e) * vby, y[1].at(e) * vby, y[2].at(e) * vby, y[3].at(e) * vby);
        if (fresh == ~0u) {
            *to = w;
        } else if (vg == 1.f) {               // bytes of their own: nothing to read first
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (fresh >> (8 * i) & 1) ((unsigned char*)to)[i] = (unsigned char)(w >> (8 * i));
        } else {
            const unsigned had = *to;
            *to = (w & fresh) | (rescaled(had, vg) & older) | (had & ~(fresh | older));
        }
    }
}

template <typename T>
static znni_status launch_append(const AppendArgs& a, int B, int max_new, const znni_heads* k, const znni_heads* v, hipStream_t st)
{
    // tokens that begin anywhere in a page reach this many
    const long long reach = ((long long)max_new + PAGE - 2) / PAGE + 1, pages = reach < a.width ? reach : a.width;
    if (pages > LAUNCH_X) return ZNNI_ERR_SHAPE;
    k_append<T><<<dim3((unsigned)pages, (unsigned)a.Hk, (unsigned)B), dim3(APPEND_THREADS), 0, st>>>(a, heads_of<const T>(k), heads_of<const T>(v));
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni

using namespace znni;

extern "C" znni_status znni_kv8_append(int type, int B, int Hk, int D, const znni_heads* k, const znni_heads* v, const int* cu,
                                       const int* start, int max_new, unsigned char* kcodes, unsigned char* vcodes, float* scales,
                                       int pages, const int* table, int width, void* stream)
{
    if (!k || !v) return ZNNI_ERR_NULL;
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (B < 0 || B > 65535 || max_new < 0 || pages < 0 || width < 0) return ZNNI_ERR_SHAPE;
    const znni_status rc = heads_shape(Hk, Hk, D);
    if (rc) return rc;
    if (B == 0 || max_new == 0 || pages == 0 || width == 0) return ZNNI_OK;
    if (!k->data || !v->data || !cu || !start || !kcodes || !vcodes || !scales || !table) return ZNNI_ERR_NULL;
    if (!heads_aligned(k, type) || !heads_aligned(v, type) || !cache_aligned(kcodes, vcodes, scales) ||
        (((uintptr_t)cu | (uintptr_t)start | (uintptr_t)table) & 3u))
        return ZNNI_ERR_ALIGN;
    const AppendArgs a = {Hk, D, pages, width, cu, start, table, kcodes, vcodes, scales};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_append<float>(a, B, max_new, k, v, st);
        case ZNNI_BF16: return launch_append<bf16>(a, B, max_new, k, v, st);
        default: return launch_append<f16>(a, B, max_new, k, v, st);
    }
}
