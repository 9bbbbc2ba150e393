// kv8.hip -- filling the 8-bit cache of keys and values.
//
// A workgroup has one page and head: it reads the tokens that come to the page (16 bytes a thread and load, kept in
// registers), takes their largest magnitude, decides the scale and writes codes, keys as they come and values through LDS
// with the tokens innermost.  Bound by memory for prompts, by the chain of dependent reads (start, table, scale, tokens) for single tokens.
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
constexpr int CHUNKS = PAGE * ATTN_DMAX / 8 / APPEND_THREADS;     // of eight values, for a thread

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

__device__ inline float block_max(float a, float* red)
{
    for (int o = 32; o; o >>= 1) a = fmaxf(a, __shfl_xor(a, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    __syncthreads();
    for (int w = 0; w < APPEND_THREADS / 64; ++w) a = fmaxf(a, red[w]);
    return a;
}

template <typename T>
struct Eight {
    T x[8];
};

template <typename T>
__device__ inline void load8(const T* p, float* f)
{
    struct alignas(16) { Eight<T> e; } v;
    const uint4* s = (const uint4*)p;
    uint4* d = (uint4*)&v;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i) d[i] = s[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v.e.x[i];
}

template <typename T>
__global__ __launch_bounds__(APPEND_THREADS) void k_append(AppendArgs a, Heads<const T> k, Heads<const T> v)
{
    __shared__ __align__(16) unsigned char turned[ATTN_DMAX * PAGE];
    __shared__ float red[APPEND_THREADS / 64];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int c0 = a.cu[b], n = a.cu[b + 1] - c0, start = a.start[b];
    const long long index = (long long)start / PAGE + blockIdx.x, base = index * PAGE;
    const int s0 = (int)(start > base ? start - base : 0);                       // slots s0 .. s1 are new, those before s0 old
    const int s1 = (int)min((long long)PAGE, (long long)start + n - base);
    if (s0 >= s1 || start < 0 || index >= a.width) return;
    const int page = a.table[(long long)b * a.width + index];
    if (page < 0 || page >= a.pages) return;
    const long long at = ((long long)page * a.Hk + h), token = c0 + base - start;
    unsigned char* kc = a.kcodes + at * PAGE * a.D;
    unsigned char* vc = a.vcodes + at * PAGE * a.D;
    const int per = a.D / 8, chunks = (s1 - s0) * per;
    // Keys, then values: at most four chunks of eight values a thread.
    for (int which = 0; which < 2; ++which) {
        const Heads<const T>& src = which ? v : k;
        float x[CHUNKS][8], top = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int i = t + c * APPEND_THREADS;
            if (i < chunks) {
                const int slot = s0 + i / per, d = i % per * 8;
                load8(src.row(token + slot, h) + d, x[c]);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = largest(top, x[c][e]);
            }
        }
        int E = exponent_of(block_max(top, red));
        float grown = 1.f;
        if (s0) {
            const float was = a.scales[at * 2 + which];
            const int before = (int)(__float_as_uint(was) >> 23 & 255) - 127;
            if (before >= E) E = before;
            else grown = power_of_two(before - E > -126 ? before - E : -126);
        }
        // every thread has read the old scale before it changes
        __syncthreads();
        if (t == 0) a.scales[at * 2 + which] = power_of_two(E);
        const float up = power_of_two(-E);          // E <= 120
        if (!which) {
            if (grown != 1.f)
                for (int i = t; i < s0 * per * 2; i += APPEND_THREADS) ((unsigned*)kc)[i] = rescaled(((unsigned*)kc)[i], grown);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int i = t + c * APPEND_THREADS;
                if (i < chunks) {
                    float* y = x[c];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= up;
                    *(uint2*)(kc + (s0 + i / per) * a.D + i % per * 8) =
                        make_uint2(codes_of(y[0], y[1], y[2], y[3]), codes_of(y[4], y[5], y[6], y[7]));
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int i = t + c * APPEND_THREADS;
                if (i < chunks) {
                    const int slot = s0 + i / per, d = i % per * 8;
                    float* y = x[c];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= up;
                    const unsigned lo = codes_of(y[0], y[1], y[2], y[3]), hi = codes_of(y[4], y[5], y[6], y[7]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) turned[(d + e) * PAGE + slot] = (unsigned char)((e < 4 ? lo : hi) >> (e % 4 * 8));
                }
            }
            __syncthreads();
            // sixteen slots of one element of the head: old ones stay (or are rescaled), new ones are set
            for (int i = t; i < a.D * (PAGE / 16); i += APPEND_THREADS) {
                const int d = i / (PAGE / 16), g = i % (PAGE / 16) * 16;
                if (g >= s1 || (g + 16 <= s0 && grown == 1.f)) continue;
                uint4* dst = (uint4*)(vc + d * PAGE + g);
                uint4 w = *(const uint4*)(turned + d * PAGE + g);
                if (g < s0 || g + 16 > s1) {
                    const uint4 old = *dst;
                    const unsigned o[4] = {old.x, old.y, old.z, old.w};
                    unsigned* y = (unsigned*)&w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned kept = grown != 1.f ? rescaled(o[e], grown) : o[e];
                        unsigned r = 0;
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            const int slot = g + e * 4 + f;
                            r |= (slot < s0 ? kept : slot < s1 ? y[e] : o[e]) & (255u << (8 * f));
                        }
                        y[e] = r;
                    }
                }
                *dst = w;
            }
        }
    }
}

template <typename T>
static znni_status launch_append(const AppendArgs& a, int B, int max_new, const znni_heads* k, const znni_heads* v, hipStream_t st)
{
    // tokens that begin anywhere in a page reach this many
    const int reach = (int)(((long long)max_new + PAGE - 2) / PAGE + 1);
    k_append<T><<<dim3((unsigned)reach, (unsigned)a.Hk, (unsigned)B), dim3(APPEND_THREADS), 0, st>>>(a, heads_of<const T>(k), heads_of<const T>(v));
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
