// rope.hip -- rotary positions with several axes: pair j of a head is turned by pos[token][axis(j)] * freq[j].
//
// Bound by memory: every value of q and k is read and written once.  The sines and cosines of a token are the same for
// all its heads: a workgroup takes whole tokens, works them out once into LDS and then walks the tokens' heads.
// bf16, 32768 tokens, heads 16 + 4 x 128, 336 MB: 58 us, 5.8 TB/s, where a large copy reaches 6.25; 8 tokens: 2.6 us, an empty kernel's time.
#include "attn_common.h"

namespace znni {

constexpr int ROPE_MAX_D = 512;          // elements of a head
constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TABLE = 1024;         // pairs (of all tokens of a workgroup) in LDS

struct RopeArgs {
    int T, Hq, Hk, D, R, axes;
    int end[ZNNI_ROPE_MAX_AXES];         // pairs below end[a] that no earlier axis has belong to axis a
    int tokens;                          // tokens of a workgroup
};

// The angle in turns, in 64 bits: positions times frequencies pass 2^24 long before they stop mattering, and the part
// below one turn is all that counts.
__device__ inline void turn_of(int pos, float freq, float* c, float* s)
{
    double t = (double)pos * (double)freq * 0.15915494309189533577;
    t -= rint(t);
    sincospif(2.0f * (float)t, s, c);
}

// VEC elements a load.  Pairs of halves: (x[j], x[R + j]), VEC divides R; neighbours: (x[2j], x[2j + 1]).
template <typename T, int VEC, bool NEIGHBOURS>
__global__ __launch_bounds__(ROPE_THREADS) void k_rope(RopeArgs a, Heads<const T> q, Heads<const T> k, const int* __restrict__ pos,
                                                       const float* __restrict__ freq, Heads<T> qo, Heads<T> ko)
{
    typedef T V __attribute__((ext_vector_type(VEC)));
    __shared__ float2 table[ROPE_TABLE];
    const long long t0 = group_id() * a.tokens;
    if (t0 >= a.T) return;
    const int nt = (int)min((long long)a.tokens, a.T - t0);
    for (int i = threadIdx.x; i < nt * a.R; i += ROPE_THREADS) {
        const int tok = i / a.R, j = i - tok * a.R;
        int ax = 0;
        while (j >= a.end[ax]) ++ax;
        float2 cs;
        turn_of(pos[(t0 + tok) * a.axes + ax], freq[j], &cs.x, &cs.y);
        table[i] = cs;
    }
    __syncthreads();
    // units of a head: with halves R / VEC pairs of vectors, then the vectors that pass; with neighbours D / VEC vectors
    const int turned = NEIGHBOURS ? a.D / VEC : a.R / VEC;
    const int units = NEIGHBOURS ? turned : turned + (a.D - 2 * a.R) / VEC;
    const int heads = a.Hq + a.Hk, n = nt * heads * units;
    for (int i = threadIdx.x; i < n; i += ROPE_THREADS) {
        const int row = i / units, u = i - row * units, tok = row / heads, h = row - tok * heads;
        const T* x = h < a.Hq ? q.row(t0 + tok, h) : k.row(t0 + tok, h - a.Hq);
        T* y = h < a.Hq ? qo.row(t0 + tok, h) : ko.row(t0 + tok, h - a.Hq);
        const float2* cs = table + tok * a.R;
        if constexpr (NEIGHBOURS) {
            V v = *(const V*)(x + u * VEC);
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const int j = (u * VEC + e) / 2;
                if (j < a.R) {
                    const float2 t = cs[j];
                    const float p = (float)v[e], r = (float)v[e + 1];
                    v[e] = (T)(p * t.x - r * t.y);
                    v[e + 1] = (T)(p * t.y + r * t.x);
                }
            }
            *(V*)(y + u * VEC) = v;
        } else if (u < turned) {
            const V v = *(const V*)(x + u * VEC), z = *(const V*)(x + a.R + u * VEC);
            V w0, w1;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 t = cs[u * VEC + e];
                const float p = (float)v[e], r = (float)z[e];
                w0[e] = (T)(p * t.x - r * t.y);
                w1[e] = (T)(p * t.y + r * t.x);
            }
            *(V*)(y + u * VEC) = w0;
            *(V*)(y + a.R + u * VEC) = w1;
        } else {
            const int at = 2 * a.R + (u - turned) * VEC;
            *(V*)(y + at) = *(const V*)(x + at);
        }
    }
}

template <typename T>
static znni_status launch_rope(RopeArgs a, bool neighbours, const znni_heads* q, const znni_heads* k, const int* pos, const float* freq,
                               const znni_heads* qo, const znni_heads* ko, hipStream_t st)
{
    constexpr int WIDE = 16 / sizeof(T);
    // Two vectors or so a thread, 32768 tokens of 20 heads of 128: 58 us (5.8 TB/s) with one to three, 61 with four, 64 with eight.
    a.tokens = ROPE_TABLE / (a.R > 0 ? a.R : 1);
    const int units = (a.Hq + a.Hk) * a.D / WIDE;
    const int want = (2 * ROPE_THREADS + units - 1) / units;
    if (a.tokens > want) a.tokens = want;
    const int spread = (int)((a.T + 1023LL) / 1024);                          // at least 1024 workgroups if there are tokens for them
    if (a.tokens > spread) a.tokens = spread;
    if (a.tokens < 1) a.tokens = 1;
    const dim3 grid = launch_of(((long long)a.T + a.tokens - 1) / a.tokens), block(ROPE_THREADS);
    const Heads<const T> qi = heads_of<const T>(q), ki = heads_of<const T>(k);
    const Heads<T> oq = heads_of<T>(qo), ok = heads_of<T>(ko);
    // Every row starts at a multiple of 16 bytes; its second half, and what passes, at a multiple of the widest vector that divides R.
    // (Wide vectors from wherever the half starts, the last one element by element, are slower: R = 44 148 us against 83, 45 200 and 178.)
    if (neighbours) k_rope<T, WIDE, true><<<grid, block, 0, st>>>(a, qi, ki, pos, freq, oq, ok);
    else if (a.R % WIDE == 0) k_rope<T, WIDE, false><<<grid, block, 0, st>>>(a, qi, ki, pos, freq, oq, ok);
    else if (WIDE > 4 && a.R % 4 == 0) k_rope<T, 4, false><<<grid, block, 0, st>>>(a, qi, ki, pos, freq, oq, ok);
    else if (a.R % 2 == 0) k_rope<T, 2, false><<<grid, block, 0, st>>>(a, qi, ki, pos, freq, oq, ok);
    else k_rope<T, 1, false><<<grid, block, 0, st>>>(a, qi, ki, pos, freq, oq, ok);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

}  // namespace znni

using namespace znni;

extern "C" znni_status znni_rope_axes(int type, int T, int Hq, int Hk, int D, const znni_heads* q, const znni_heads* k, const int* pos,
                                      const float* freq, int axes, const int* sections, const znni_heads* q_out,
                                      const znni_heads* k_out, unsigned flags, void* stream)
{
    if (!q || !q_out || !sections || (Hk > 0 && (!k || !k_out))) return ZNNI_ERR_NULL;
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (flags & ~ZNNI_ROPE_NEIGHBOURS) return ZNNI_ERR_FLAGS;
    if (T < 0 || Hq < 1 || Hk < 0 || Hq > 65535 || Hk > 65535 || D < 1 || axes < 1) return ZNNI_ERR_SHAPE;
    if (D % 8 || D > ROPE_MAX_D || axes > ZNNI_ROPE_MAX_AXES) return ZNNI_ERR_UNSUPPORTED_SIZE;
    RopeArgs a = {};
    a.T = T; a.Hq = Hq; a.Hk = Hk; a.D = D; a.axes = axes;
    for (int x = 0; x < axes; ++x) {
        if (sections[x] < 0 || sections[x] > D) return ZNNI_ERR_SHAPE;
        a.R += sections[x];
        a.end[x] = a.R;
    }
    if (2 * a.R > D) return ZNNI_ERR_SHAPE;
    if (T == 0) return ZNNI_OK;
    if (!q->data || !q_out->data || (Hk > 0 && (!k->data || !k_out->data)) || (a.R > 0 && (!pos || !freq))) return ZNNI_ERR_NULL;
    const znni_heads none = {nullptr, 0, 0};
    if (Hk == 0) k = k_out = &none;
    if (((uintptr_t)pos | (uintptr_t)freq) & 3u) return ZNNI_ERR_ALIGN;
    for (const znni_heads* h : {q, k, q_out, k_out})
        if (!heads_aligned(h, type)) return ZNNI_ERR_ALIGN;
    const hipStream_t st = (hipStream_t)stream;
    const bool nb = flags & ZNNI_ROPE_NEIGHBOURS;
    switch (type) {
        case ZNNI_F32: return launch_rope<float>(a, nb, q, k, pos, freq, q_out, k_out, st);
        case ZNNI_BF16: return launch_rope<bf16>(a, nb, q, k, pos, freq, q_out, k_out, st);
        default: return launch_rope<f16>(a, nb, q, k, pos, freq, q_out, k_out, st);
    }
}
