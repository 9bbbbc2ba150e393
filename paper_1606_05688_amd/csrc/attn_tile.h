// attn_tile.h -- windowed attention: what a workgroup's rows see, key tiles in LDS, and the matrix instructions on them.
#pragma once
#include "attn_common.h"

namespace znni {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    int Hq, Hk, D;
    const int* cu_q;
    const int* cu_k;
    Window w;
    float scale;
    int groups, max_q;
    int tiles, splits, tile_rows;     // row tiles of a sequence, workgroups that share a tile's keys, rows of a tile in `parts`
    float* parts;
    float2* stats;
};

template <typename T, int NC, int THREADS>
struct AttnTile {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int BN = F32 ? 32 : 64;                       // keys
    static constexpr int EC = 16 / sizeof(T);                      // elements of a 16-byte chunk
    static constexpr int RS = NC == 3 ? 128 : 32 * NC;             // elements of a row in LDS
    static constexpr int CR = RS / EC;                             // its chunks
    static constexpr int PER = BN * CR / THREADS;                  // chunks a thread brings
    static constexpr int STAGES = NC == 1 ? 4 : NC == 2 ? 3 : 2;   // tiles in LDS: what leaves two workgroups a compute unit, or three
    // Chunk c of key j lies at c ^ swizzle(j).  Scores read one chunk of 32 keys, 16 bytes a lane: 256 bytes of
    // consecutive keys get different places; values read, 16-bit: four keys, 64 bytes each, fp32: two keys four apart, 128 bytes each.
    __device__ static int swizzle_k(int j) { return CR >= 16 ? j & 15 : CR == 8 ? j >> 1 & 7 : j >> 2 & 3; }
    __device__ static int swizzle_v(int j)
    {
        if (F32) return CR >= 16 ? (j >> 2 & 1) << 3 : 0;
        return CR == 16 ? (j & 3) << 2 : CR == 8 ? (j >> 1 & 1) << 2 : 0;
    }
};

// An address that is the same for all lanes, in scalar registers.
__device__ inline const void* uniform(const void* p)
{
    const unsigned long long x = (unsigned long long)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
    return (const void*)((unsigned long long)hi << 32 | lo);
}

// (The compiler keeps m0 for itself and warns of its name in the lists below, which is what tells it not to count on m0 across them.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes a lane from memory to LDS, 1024 bytes of a wave from `lds` on.  As assembly, since the compiler, which sees one
// array in LDS, waits for such a load before any read of it: wait_but_and_meet() is what waits for these.
__device__ inline void to_lds(const void* base, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset),
                 "s"(uniform(base)) : "m0", "memory");
}
__device__ inline void to_lds(const void* from, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ inline unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// Four elements of one column of four rows: lanes 4r .. 4r + 3 of sixteen bring row r, lane c of them gets column c.
template <typename V4>
__device__ inline V4 transposed(const char* p)
{
    return __builtin_bit_cast(V4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

// All loads but the LEFT newest have come, for all waves.
template <int LEFT>
__device__ inline void wait_but_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// What this wave wrote to LDS is there for all (loads into LDS go on).
__device__ inline void wait_and_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {
    typedef bf16 V __attribute__((ext_vector_type(8)));
    typedef bf16 V4 __attribute__((ext_vector_type(4)));
    __device__ static f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<f16> {
    typedef f16 V __attribute__((ext_vector_type(8)));
    typedef f16 V4 __attribute__((ext_vector_type(4)));
    __device__ static f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<float> {
    typedef float V __attribute__((ext_vector_type(4)));
    __device__ static f32x16 mul(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
};

// What kind of number x is, so that a sum of up to 64 says which kinds were there: 1 for infinity, 128 for minus infinity, both for NaN, 0 else.
__device__ inline float kind_of(float x)
{
    return fabsf(x) <= 3.402823466e38f ? 0.f : x == INFINITY ? 1.f : x == -INFINITY ? 128.f : 129.f;
}

// What rows at positions p0 .. p1 (none if p1 < p0) see of nk keys: the first row's keys go from lo0 to hi0, the last one's from lo1
// to hi1, besides sinks.
struct Sight {
    int lo0, hi0, lo1, hi1, sinks;
    __device__ Sight(long long p0, long long p1, int nk, const Window& w) : sinks(w.sinks)
    {
        window_of(p0, nk, w, &lo0, &hi0);
        window_of(p1, nk, w, &lo1, &hi1);
        if (p1 < p0) hi0 = hi1 = -1;
    }
    __device__ bool all(int j0, int n) const { return j0 + n - 1 <= hi0 && (j0 >= lo1 || j0 + n <= sinks); }
    __device__ bool any(int j0, int n) const { return j0 <= hi1 && (j0 + n - 1 >= lo0 || j0 < sinks); }
};

// Their key tiles: those of sinks alone, then those of the window.
template <int BN>
struct KeyTiles {
    int sink_tiles, first, n;
    __device__ KeyTiles(const Sight& s)
    {
        first = s.lo0 / BN;
        sink_tiles = min((min(s.sinks, s.hi1 + 1) + BN - 1) / BN, first);
        n = s.hi1 < s.lo0 ? sink_tiles : sink_tiles + s.hi1 / BN - first + 1;
    }
    __device__ int base(int i) const { return (i < sink_tiles ? i : first + i - sink_tiles) * BN; }
};

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: runs of eight neighbouring row tiles, which see nearly the
// same keys, to the same one (16384 tokens, window of 4096: 647 us in turn, 613 in runs of 4, 610 of 8, 625 of 16, 647 of 32).
__device__ inline int in_runs(int id, int n)
{
    return id < n / 64 * 64 ? (id / 64 * 8 + id % 8) * 8 + id / 8 % 8 : id;
}

}  // namespace znni
