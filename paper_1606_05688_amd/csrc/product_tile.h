// product_tile.h -- tiles of two matrices in LDS and their product on the matrix cores, for sums over either index of each.
#pragma once
#include "attn_tile.h"
#include "rows_common.h"

namespace znni {

// What lanes of this wave wrote to LDS is there for its other lanes, what they read there may be written over.  (The hardware keeps a wave's
// accesses in order; this is what keeps the compiler from moving them past each other.)
__device__ inline void wave_meets()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// A matrix in device memory as one side of a product: element (row r of the result's side, c of the sum) lies at p[r * ld + c] if
// the sum's index is the contiguous one, at p[c * ld + r] if not.
template <typename T>
struct Side {
    const T* p;
    long long ld;
    int rows;
    bool wide;            // direct loads of 16 bytes: address and rows are aligned
};

// ROWS rows by BK steps of the sum in LDS, in chunks of 16 bytes.  SUM_INNER: rows of 8 chunks along the sum; else BK rows of the
// matrix as they stand.  Chunks of a row are permuted so that neither kind of read meets a bank twice.
template <typename T, bool SUM_INNER, int ROWS, int THREADS>
struct Tile {
    static constexpr int EC = 16 / sizeof(T), BK = 8 * EC;
    static constexpr int CR = SUM_INNER ? 8 : ROWS / EC;
    static constexpr int PER = ROWS * 8 / THREADS;              // chunks a thread brings
    static constexpr unsigned BYTES = ROWS * 128;
    __device__ static int swizzle(int j)
    {
        if (SUM_INNER) return j >> 1 & 7;
        if (sizeof(T) == 4) return CR >= 16 ? (j >> 2 & 1) << 3 : 0;
        return CR >= 16 ? (j & 3) << 2 : (j >> 1 & 1) << 2;
    }
    typedef T Chunk __attribute__((ext_vector_type(EC)));

    unsigned at[PER];           // where this thread's chunks lie, from the tile's first element on
    bool plain;                 // whole tiles come by direct loads
    __device__ void find(const Side<T>& s, int row0, int t)
    {
        // (offsets of 32 bits: a tile spans at most 256 rows of the matrix)
        plain = s.wide && s.ld >= 0 && s.ld < 1 << 21 && (SUM_INNER || s.rows % EC == 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int slot = i * THREADS + t, j = slot / CR, c = (slot % CR ^ swizzle(j)) * EC;
            // rows past the last: the last again, whose products nobody keeps
            const int r = SUM_INNER ? min(j, s.rows - 1 - row0) : j, e = SUM_INNER ? c : max(0, min(c, s.rows - EC - row0));
            at[i] = ((unsigned)r * (unsigned)s.ld + (unsigned)e) * (unsigned)sizeof(T);
        }
    }
    // Steps k0 .. of the sum, those from `end` on as zeros.  Direct loads are in flight afterwards, PER of them or none.
    __device__ void bring(const Side<T>& s, int row0, int k0, int end, char* lds, int t)
    {
        if (plain && k0 + BK <= end) {
            const T* base = SUM_INNER ? s.p + row0 * s.ld + k0 : s.p + k0 * s.ld + row0;
            const unsigned to = lds_address(lds) + (unsigned)__builtin_amdgcn_readfirstlane(t >> 6) * 1024;
#pragma unroll
            for (int i = 0; i < PER; ++i) to_lds(base, at[i], to + i * THREADS * 16);
            return;
        }
        if (plain && (!SUM_INNER || (end - k0) % EC == 0)) {
            // the last steps, in whole chunks: direct loads of those that are there
            const T* base = SUM_INNER ? s.p + row0 * s.ld + k0 : s.p + k0 * s.ld + row0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int slot = i * THREADS + t, j = slot / CR;
                if (k0 + (SUM_INNER ? (slot % CR ^ swizzle(j)) * EC : j) < end)
                    to_lds((const char*)base + at[i], lds_address(lds) + (unsigned)__builtin_amdgcn_readfirstlane(t >> 6) * 1024 + i * THREADS * 16);
                else *(uint4*)(lds + slot * 16) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            return;
        }
        Chunk y[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int slot = i * THREADS + t, j = slot / CR, c = (slot % CR ^ swizzle(j)) * EC;
            const int r = SUM_INNER ? row0 + j : row0 + c, k = SUM_INNER ? k0 + c : k0 + j;
            const T* p = SUM_INNER ? s.p + r * s.ld + k : s.p + k * s.ld + r;
            // how many elements are there
            const int n = SUM_INNER ? (r < s.rows ? end - k : 0) : (k < end ? s.rows - r : 0);
            y[i] = Loose<T, EC>::load(p, n);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) *(Chunk*)(lds + (i * THREADS + t) * 16) = y[i];
        // (direct loads of earlier tiles are counted by wait_but_and_meet: none may be left that it does not know of)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }

    // Operand of 32 rows from `row` on in step c: 16 steps of the sum (8 a lane) or, in fp32, 8 (4 a lane).
    __device__ static typename Mfma<T>::V operand(const char* lds, int row, int c, int l)
    {
        using M = Mfma<T>;
        const int h = l >> 5, c32 = l & 31;
        if constexpr (SUM_INNER) {
            const int j = row + c32;
            return *(const typename M::V*)(lds + j * 128 + ((2 * c + h) ^ swizzle(j)) * 16);
        } else if constexpr (sizeof(T) == 4) {
            typename M::V y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 8 * c + 4 * h + e;
                y[e] = *(const T*)(lds + j * (CR * 16) + (((row + c32) / EC) ^ swizzle(j)) * 16 + (c32 & 3) * 4);
            }
            return y;
        } else {
            const int j = 16 * c + 8 * h + (l >> 2 & 3), x = row + (l >> 4 & 1) * 16 + (l & 3) * 4;
            const char* p = lds + j * (CR * 16) + ((x / EC) ^ swizzle(j)) * 16 + (x & 4) * 2;
            const char* p4 = lds + (j + 4) * (CR * 16) + ((x / EC) ^ swizzle(j + 4)) * 16 + (x & 4) * 2;
            const typename M::V4 y0 = transposed<typename M::V4>(p), y1 = transposed<typename M::V4>(p4);
            return __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

}  // namespace znni
