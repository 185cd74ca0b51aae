// 64 tokens of one head in shared memory as 16-bit values, and their way into a page: what the append and the eviction share.
#ifndef SPQT_KV_TILE_HPP
#define SPQT_KV_TILE_HPP

#include "kv_common.hpp"

namespace spqt {
namespace kv {

constexpr int kTileThreads = 256;

// The 16 fours of tokens that a wavefront takes at once are in 8 banks of 8, two in each, with four numbers behind every token.
template <int D>
struct Tile {
    uint16_t v[kBlock][D + 4];
    uint32_t largest[kTileThreads / 64];

    __device__ __forceinline__ void put(int t, int d, u32x4 x) {
        u32x2 *to = reinterpret_cast<u32x2 *>(&v[t][d]);
        to[0] = u32x2{x.x, x.y};
        to[1] = u32x2{x.z, x.w};
    }
};

// The larger magnitudes of two pairs of 16-bit numbers, as bits (both types order as their magnitude bits do).
__device__ __forceinline__ uint32_t larger_pair(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7FFF7FFFu), __builtin_bit_cast(u16x2, b & 0x7FFF7FFFu)));
}
// The largest number of all threads'.
template <int D>
__device__ __forceinline__ uint32_t largest_number(Tile<D> &tile, uint32_t m) {
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
// The largest magnitude (16 bits) of all threads' pairs.
template <int D>
__device__ __forceinline__ uint32_t largest_of(Tile<D> &tile, uint32_t pair) {
    return largest_number(tile, (pair & 0x7FFFu) > (pair >> 16 & 0x7FFFu) ? (pair & 0x7FFFu) : (pair >> 16 & 0x7FFFu));
}

// The lower or upper one of two numbers.
template <bool BF16>
__device__ __forceinline__ float half_of(uint32_t pair, int upper) {
    if (BF16) return as_float(upper ? pair & 0xFFFF0000u : pair << 16);
    return widen<false>((uint16_t)(upper ? pair >> 16 : pair & 0xFFFFu));
}

// Quantizes tokens from .. to - 1 of the tile into the page.  code(pair, upper, t): the stored byte, in the lowest bits of a number, of the lower or upper one of two elements of token t.
template <int D, class F>
__device__ __forceinline__ void store_codes(const Cache &c, const Tile<D> &tile, uint32_t page, int head, int which, int from, int to, float scale, F code) {
    uint8_t *out = c.codes + codes_at(c, page, head, which);
    if (which == 0) {
        for (int p = from * (D / 16) + (int)threadIdx.x; p < to * (D / 16); p += kTileThreads) {
            const u32x2 *x = reinterpret_cast<const u32x2 *>(&tile.v[p / (D / 16)][p % (D / 16) * 16]);
            uint32_t c[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = code(x[i / 4][i / 2 % 2], i % 2, p / (D / 16));
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = bytes_of(c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3], scale);
            *reinterpret_cast<u32x4 *>(out + p * 16) = w;
        }
        return;
    }
    if (from == 0 && to == kBlock) {                      // sixteen tokens of two elements at a time
        for (int p = (int)threadIdx.x; p < D * 2; p += kTileThreads) {
            const int d = p / 4 * 2, quarter = p % 4;
            u32x4 w[2];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                uint32_t x[4];
                const int t = 16 * n + 4 * quarter;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint32_t *>(&tile.v[t + i][d]);
#pragma unroll
                for (int e = 0; e < 2; ++e) w[e][n] = bytes_of(code(x[0], e, t), code(x[1], e, t + 1), code(x[2], e, t + 2), code(x[3], e, t + 3), scale);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) *reinterpret_cast<u32x4 *>(out + (d + e) * kBlock + 16 * quarter) = w[e];
        }
        return;
    }
    // four tokens of two elements at a time
    for (int p = (int)threadIdx.x; p < D * 8; p += kTileThreads) {
        const int d = p / 16 * 2, word = p % 16, t = word % 4 * 16 + word / 4 * 4;  // place 4 * word holds tokens t .. t + 3
        if (t + 4 <= from || t >= to) continue;
        uint32_t x[4], w[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint32_t *>(&tile.v[t + i][d]);
#pragma unroll
        for (int e = 0; e < 2; ++e) w[e] = bytes_of(code(x[0], e, t), code(x[1], e, t + 1), code(x[2], e, t + 2), code(x[3], e, t + 3), scale);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            uint8_t *at = out + (d + e) * kBlock + word * 4;
            if (t >= from && t + 4 <= to) {
                *reinterpret_cast<uint32_t *>(at) = w[e];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t + i >= from && t + i < to) at[i] = (uint8_t)(w[e] >> (8 * i));
            }
        }
    }
}

// The same of 16-bit values.
template <int D, bool BF16>
__device__ __forceinline__ void store_tile(const Cache &c, const Tile<D> &tile, uint32_t page, int head, int which, int from, int to, float scale) {
    const float inverse = 1.0f / scale;
    store_codes(c, tile, page, head, which, from, to, scale, [&](uint32_t pair, int upper, int) { return coded(half_of<BF16>(pair, upper), inverse); });
}

}  // namespace kv
}  // namespace spqt
#endif
