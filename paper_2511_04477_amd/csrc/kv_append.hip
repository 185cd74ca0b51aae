// spqt_kv_append: new tokens into the pages, 8 bits with a scale per block, head and side; spqt_kv_read: back to 16 bits.
#include "kv_tile.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

// code = x / scale to the nearest integer, scale = scale_of(the largest |x| of the block's tokens and head), which is known only when all of them are there: a block goes through
// shared memory once.
// One workgroup per block that the call writes to, head and side (keys or values), the heads of a token one after the other as they lie in memory: with the blocks first instead,
// 79.0 for 76.6 us below, since a line of DRAM has several heads of a token.  The first workgroup does the sequence's first and last block, one after the other, since the first
// reads from the tail what the last one overwrites there.
// What bounds it: 2 bytes in and 1 out a value, and that a workgroup's loads, largest magnitude and stores follow each other: 25.7k tokens of 8 heads of 128 (6 sequences, 158 MB)
// 47 us = 3.4 TB/s (a copy: 4.83).  With 79 registers a CU holds six workgroups; eight would take 16 of them to scratch memory.  One token of 4 sequences 5.2 us: the chain lengths, table, row,
// magnitude, codes.
template <int D, bool BF16>
__global__ __launch_bounds__(kTileThreads) void spqt_kv_append_kernel(Cache c, Rows keys, Rows values, int rows, const int32_t *counts) {
    __shared__ Tile<D> tile;
    const int s = blockIdx.z, head = blockIdx.x >> 1, which = blockIdx.x & 1;
    const int length = length_of(c, s), count = count_of(counts, s, rows);
    if (length == 0 || count == 0) return;
    const int row0 = length - count, start = row0 < 0 ? 0 : row0;             // position of row 0, and of the first token that there is
    const int first = block_of(start), last = block_of(length - 1);
    const Rows r = which ? values : keys;
    const uint16_t *in = r.data + s * r.sequence + head * r.head;
    uint16_t *tail = c.tail + (((size_t)s * c.kv_heads + head) * 2 + which) * (size_t)(kBlock * D);
    const int32_t *table = c.table + (size_t)s * c.max_blocks;

    int block = first + (int)blockIdx.y;
    if (blockIdx.y > 0 && block >= last) return;
    for (;;) {
        const int base = block * kBlock;
        const int from = start > base ? start - base : 0, to = length - base < kBlock ? length - base : kBlock;
        const uint32_t page = (uint32_t)table[block];
        const bool there = page < c.pages;
        uint32_t pair = 0;
        u32x4 x[D / 32];
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            const int p = (int)threadIdx.x + n * kTileThreads, t = p / (D / 8);
            if (t >= from && t < to) x[n] = *reinterpret_cast<const u32x4 *>(in + (base + t - row0) * r.row + p % (D / 8) * 8);
        }
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            const int p = (int)threadIdx.x + n * kTileThreads, t = p / (D / 8);
            if (t < from || t >= to) continue;
            tile.put(t, p % (D / 8) * 8, x[n]);
            pair = larger_pair(larger_pair(pair, x[n].x), larger_pair(x[n].y, larger_pair(x[n].z, x[n].w)));
            if (block == last && to < kBlock) *reinterpret_cast<u32x4 *>(tail + p * 8) = x[n];
        }
        const float fresh = scale_of<BF16>(largest_of(tile, pair));
        if (there) {
            float *scales = c.scales + scale_at(c, page, head, which);
            const float held = from > 0 ? *scales : 0.0f;
            const float scale = held != held || fresh != fresh ? __builtin_nanf("") : __builtin_fmaxf(held, fresh);
            const bool grown = from > 0 && !(scale == held);
            if (grown)
                for (int p = (int)threadIdx.x; p < from * (D / 8); p += kTileThreads)
                    tile.put(p / (D / 8), p % (D / 8) * 8, *reinterpret_cast<const u32x4 *>(tail + p * 8));
            __syncthreads();                       // the tile is whole, and everyone has the old scale
            store_tile<D, BF16>(c, tile, page, head, which, grown ? 0 : from, to, scale);
            if (threadIdx.x == 0) *scales = scale;
            if (which == 0 && c.weights && (int)threadIdx.x >= from && (int)threadIdx.x < to) c.weights[weight_at(c, page, head) + threadIdx.x] = 0.0f;
        }
        if (blockIdx.y > 0 || block == last) return;
        block = last;
        __syncthreads();                           // the tile is free again
    }
}

// x = code * scale, rounded to the rows' type: the only rounding.
// One workgroup per block that the call reads from, head and side.  Keys go straight through; values go through shared memory as they are, and come out
// four tokens of eight elements at a time, so that a row's elements leave 16 bytes a lane.
// What bounds it: 1 byte in and 2 out a value: the same 25.7k tokens (158 MB, and 42 MB of rows that it clears) 30.4 us = 6.6 TB/s; one token of 4 sequences 3.7 us.
template <int D, bool BF16>
__global__ __launch_bounds__(kTileThreads) void spqt_kv_read_kernel(Cache c, Rows keys, Rows values, int rows, const int32_t *counts) {
    constexpr int kLine = kBlock / 4 + 1;                 // words of an element's tokens, and one
    __shared__ uint32_t codes[D * kLine];
    const int s = blockIdx.z, head = blockIdx.x >> 1, which = blockIdx.x & 1;
    const int length = length_of(c, s), count = count_of(counts, s, rows), row0 = length - count;
    const int block = block_of(row0) + (int)blockIdx.y, base = block * kBlock;
    if (base - row0 >= rows) return;
    const Rows r = which ? values : keys;
    uint16_t *out = r.data + s * r.sequence + head * r.head;
    const bool any = block >= 0 && base < length;
    uint32_t page = any ? (uint32_t)c.table[(size_t)s * c.max_blocks + block] : 0u;
    const bool there = page < c.pages;
    if (!there) page = 0;
    const float scale = there ? c.scales[scale_at(c, page, head, which)] : __builtin_nanf("");
    const uint8_t *in = c.codes + codes_at(c, page, head, which);
    auto write = [&](int t, int d, u32x2 bytes) {
        const int i = base + t - row0;
        if (i < 0 || i >= rows) return;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (i < count && base + t >= 0)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = values_of<BF16>(bytes[j / 2] >> (16 * (j % 2)) & 255, bytes[j / 2] >> (16 * (j % 2) + 8) & 255, scale);
        *reinterpret_cast<u32x4 *>(out + i * r.row + d) = x;
    };
    if (which == 0) {
#pragma unroll
        for (int p = (int)threadIdx.x; p < kBlock * (D / 8); p += kTileThreads)
            write(p / (D / 8), p % (D / 8) * 8, *reinterpret_cast<const u32x2 *>(in + p * 8));
        return;
    }
    for (int p = (int)threadIdx.x; p < D * 4; p += kTileThreads) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(in + p * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[p / 4 * kLine + p % 4 * 4 + i] = x[i];
    }
    __syncthreads();
    for (int p = (int)threadIdx.x; p < 16 * (D / 8); p += kTileThreads) {
        const int word = p / (D / 8), d = p % (D / 8) * 8, t = word % 4 * 16 + word / 4 * 4;
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = codes[(d + j) * kLine + word];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x2 bytes = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j) bytes[j / 4] |= (x[j] >> (8 * i) & 255u) << (8 * (j % 4));
            write(t + i, d, bytes);
        }
    }
}

int check_call(const spqt_kv_cache *cache, bool tail, const spqt_kv_rows *k, const spqt_kv_rows *v, int rows, const int32_t *counts) {
    int rc = check_cache(cache, tail);
    if (rc == SPQT_OK) rc = check_rows(k);
    if (rc == SPQT_OK) rc = check_rows(v);
    if (rc != SPQT_OK) return rc;
    if (rows < 1 || rows > kMaxRows) return SPQT_ESHAPE;
    return (uintptr_t)counts % 4 != 0 ? SPQT_EALIGN : SPQT_OK;
}

}  // namespace

extern "C" int spqt_kv_append(const spqt_kv_cache *cache, const spqt_kv_rows *k, const spqt_kv_rows *v, int rows, const int32_t *counts, void *stream) {
    const int rc = check_call(cache, true, k, v, rows, counts);
    if (rc != SPQT_OK) return rc;
    const int most = (rows + kBlock - 2) / kBlock + 1;                    // blocks that `rows` tokens can lie in
    const dim3 grid(2 * cache->kv_heads, most > 2 ? most - 1 : 1, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        hipLaunchKernelGGL((spqt_kv_append_kernel<decltype(dim)::value, decltype(bf16)::value>), grid, dim3(kTileThreads), 0, (hipStream_t)stream, view(*cache),
                           view(*k), view(*v), rows, counts);
    });
    return launched();
}

extern "C" int spqt_kv_read(const spqt_kv_cache *cache, const spqt_kv_rows *k_out, const spqt_kv_rows *v_out, int rows, const int32_t *counts, void *stream) {
    const int rc = check_call(cache, false, k_out, v_out, rows, counts);
    if (rc != SPQT_OK) return rc;
    const dim3 grid(2 * cache->kv_heads, (rows + kBlock - 2) / kBlock + 1, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        hipLaunchKernelGGL((spqt_kv_read_kernel<decltype(dim)::value, decltype(bf16)::value>), grid, dim3(kTileThreads), 0, (hipStream_t)stream, view(*cache),
                           view(*k_out), view(*v_out), rows, counts);
    });
    return launched();
}
