// back_parts.h -- gradients of windowed attention: where the sums of workgroups that share a tile's walk lie.
#pragma once
#include <hip/hip_runtime.h>

namespace znni {

constexpr int BACK_LANES = 128;           // keys (or rows) of a tile
constexpr int FAR_LANES = 32;             // keys of a far workgroup

// Of a sequence and key head (`bh`): the tiles' own parts, BACK_LANES keys (or rows) each -- of all tiles where a tile's walk is split, else of
// those that hold first tokens --, then the far workgroups', FAR_LANES keys each.  In 64 bits: 2^25 first tokens with 64 far workgroups
// a tile have 2^31 keys in parts.
struct BackParts {
    int tiles, splits;                    // tiles of keys (or rows) of a sequence, workgroups that share a tile's walk
    int first_tiles;                      // of keys: tiles that hold first tokens, which rows past their window see too:
    int far_tiles, far;                   // 32 keys at a time, so many workgroups that walk those rows
    __host__ __device__ long long owns() const { return splits > 1 ? (long long)tiles * splits : first_tiles; }
    __host__ __device__ long long per_head() const { return owns() * BACK_LANES + (long long)far_tiles * far * FAR_LANES; }
    // The first key (or row) of a part.
    __host__ __device__ long long own_part(int bh, int tile, int split) const { return bh * per_head() + ((long long)tile * splits + split) * BACK_LANES; }
    __host__ __device__ long long far_part(int bh, int tile, int split) const
    {
        return bh * per_head() + owns() * BACK_LANES + ((long long)tile * far + split) * FAR_LANES;
    }
};

}  // namespace znni
