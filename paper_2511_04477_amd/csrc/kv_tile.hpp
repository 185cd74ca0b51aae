// 64 tokens of one head in shared memory as 16-bit values, and their way into a page: what the append and the eviction share.
#ifndef SPQT_KV_TILE_HPP
#define SPQT_KV_TILE_HPP

#include "kv_common.hpp"

namespace spqt {
namespace kv {

constexpr int kTileThreads = 256;

template <int D>
struct Tile {
    uint16_t v[kBlock][D + 8];
    uint32_t largest[kTileThreads / 64];
};

// The larger magnitudes of two pairs of 16-bit numbers, as bits (both types order as their magnitude bits do).
__device__ __forceinline__ uint32_t larger_pair(uint32_t a, uint32_t b) {
    const uint32_t al = a & 0x7FFFu, ah = a & 0x7FFF0000u, bl = b & 0x7FFFu, bh = b & 0x7FFF0000u;
    return (al > bl ? al : bl) | (ah > bh ? ah : bh);
}
// The largest magnitude (16 bits) of all threads' pairs.
template <int D>
__device__ __forceinline__ uint32_t largest_of(Tile<D> &tile, uint32_t pair) {
    uint32_t m = (pair & 0x7FFFu) > (pair >> 16 & 0x7FFFu) ? (pair & 0x7FFFu) : (pair >> 16 & 0x7FFFu);
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) {
        const uint32_t other = (uint32_t)__shfl_xor((int)m, step);
        m = other > m ? other : m;
    }
    if ((threadIdx.x & 63) == 0) tile.largest[threadIdx.x >> 6] = m;
    __syncthreads();
    m = tile.largest[0];
#pragma unroll
    for (int w = 1; w < kTileThreads / 64; ++w) m = tile.largest[w] > m ? tile.largest[w] : m;
    return m;
}

// Quantizes tokens from .. to - 1 of the tile into the page.
template <int D, bool BF16>
__device__ __forceinline__ void store_tile(const Cache &c, const Tile<D> &tile, uint32_t page, int head, int which, int from, int to, float scale) {
    const float inverse = 1.0f / scale;
    uint8_t *out = c.codes + codes_at(c, page, head, which);
    if (which == 0) {
        for (int p = from * (D / 8) + (int)threadIdx.x; p < to * (D / 8); p += kTileThreads) {
            const uint16_t *x = &tile.v[p / (D / 8)][p % (D / 8) * 8];
            u32x2 w = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i / 4] |= code_of(widen<BF16>(x[i]), inverse) << (8 * (i % 4));
            *reinterpret_cast<u32x2 *>(out + p * 8) = w;
        }
        return;
    }
    for (int p = (int)threadIdx.x; p < D * 16; p += kTileThreads) {
        const int d = p / 16, word = p % 16, t = word % 4 * 16 + word / 4 * 4;      // place 4 * word holds tokens t .. t + 3
        if (t + 4 <= from || t >= to) continue;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= code_of(widen<BF16>(tile.v[t + i][d]), inverse) << (8 * i);
        if (t >= from && t + 4 <= to) {
            *reinterpret_cast<uint32_t *>(out + p * 4) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i >= from && t + i < to) out[p * 4 + i] = (uint8_t)(w >> (8 * i));
        }
    }
}

}  // namespace kv
}  // namespace spqt
#endif
