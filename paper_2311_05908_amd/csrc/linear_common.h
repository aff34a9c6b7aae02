// What the projections in 8 bits share (linear_i8.hip, linear_f8.hip): places in their results, loads of rows of bytes, stores of whole lines, the
// order of the tiles.
#pragma once

#include "async_lds.h"

namespace fftconv {
namespace lay {

// x / d for 0 <= x < 2^31 from the reciprocal: at most one too large before the correction.
__device__ __forceinline__ int quotient(int x, int d, uint32_t by_d)
{
    if (d == 1) return x;
    const uint32_t q = __umulhi((uint32_t)x, by_d);
    return (int)(q - (q * (uint32_t)d > (uint32_t)x ? 1 : 0));
}
static uint32_t reciprocal(int64_t d) { return d > 1 ? (uint32_t)((((int64_t)1 << 32) + d - 1) / d) : 0; }

// 16 bytes of a row of K from column k on; what lies beyond K reads as zero. The row's end is its last 16 bytes, moved down (a load for every byte: a product of
// 5950 x 63 -> 10176 took 141 us instead of 83).
__device__ __forceinline__ uint4 load16(const void *bytes, int64_t k, int64_t K)
{
    const uint8_t *const row = (const uint8_t *)bytes;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K && K >= 16) {
        uint64_t w[2];
        __builtin_memcpy(w, row + K - 16, 16);
        const int past = (int)(k + 16 - K) * 8;              // bits, 8 ... 120
        const uint64_t lo = past < 64 ? w[0] >> past | w[1] << (64 - past) : w[1] >> (past - 64), hi = past < 64 ? w[1] >> past : 0;
        v = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
    } else if (k < K) {
        uint32_t w[4] = {};
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (k + e < K) w[e / 4] |= (uint32_t)row[k + e] << (8 * (e % 4));
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

// The place in LDS of 16-byte piece c (0 .. 3) of a 64-byte row. A clock delivers 256 bytes, here the same piece of sixteen rows in a run: four rows
// lie in 256 bytes, so the piece is moved by the row's number above that, and all sixteen come from banks of their own.
__device__ __forceinline__ int piece_at(int row, int c) { return row * 64 + ((c ^ ((row >> 2) & 3)) << 4); }

// 16 bytes to y. Past the caches where y would only push everything else out of the memory-side one: bf16 64 x 4096 x 768 -> 3 x 768, 1.2 GB, 643 -> 619 us;
// f16 8192 x 4096 -> 16384, 0.27 GB, 505 us with and 512 without them.
template <bool BEYOND> __device__ __forceinline__ void put16(char *to, uint4 v)
{
    typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4;
    const u32x4 w = {v.x, v.y, v.z, v.w};
    if constexpr (BEYOND) __builtin_nontemporal_store(w, (u32x4 *)to);
    else *(u32x4 *)to = w;
}

// Which tile: workgroups go to the dies in turn; a die takes a stretch of the tiles, its workgroups side by side, in an order in which
// neighbours share rows of R or of S, so that those come from its L2.
struct Walk {
    int tiles_s, group, tiles;
    __device__ __forceinline__ void place(int i, int &tr, int &ts, int tiles_r) const
    {
        const int whole = tiles_r * group, g = i / whole, k = i - g * whole, width = min(group, tiles_s - g * group);
        tr = k / width, ts = g * group + (k - tr * width);
    }
};

}  // namespace lay
}  // namespace fftconv
