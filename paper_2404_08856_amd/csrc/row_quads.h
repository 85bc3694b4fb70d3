// Rows of float32 entries read 4 at a time (accept step, sampler, log probabilities).
#pragma once
#include "common.h"

namespace spd {

// Quad q of a row (entries 4 q .. 4 q + 3), `fill` beyond its end.  ALIGNED: the row is 16-byte aligned and a multiple of 4
// long.  Otherwise it starts at any multiple of 4 bytes and may end with a part of a quad: 16-byte accesses of that
// alignment, entry by entry at the end (which costs 1 us for one sequence and 4 for 64, so the two are kept apart).
struct __attribute__((packed, aligned(4))) Quad { float x, y, z, w; };
template <bool ALIGNED>
__device__ __forceinline__ float4 load_quad(const float *__restrict__ row, int q, int V, float fill) {
    if (ALIGNED) return 4 * q < V ? reinterpret_cast<const float4 *>(row)[q] : float4{fill, fill, fill, fill};
    const int left = V - 4 * q;
    if (left >= 4) {
        const Quad v = *reinterpret_cast<const Quad *>(row + 4 * q);
        return float4{v.x, v.y, v.z, v.w};
    }
    float4 v = {fill, fill, fill, fill};
    if (left > 0) v.x = row[4 * q];
    if (left > 1) v.y = row[4 * q + 1];
    if (left > 2) v.z = row[4 * q + 2];
    return v;
}

}  // namespace spd
