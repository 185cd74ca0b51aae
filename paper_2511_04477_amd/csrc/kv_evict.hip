// spqt_kv_evict: what a sequence's heads keep, and its way to other pages.
#include "kv_tile.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

constexpr int kSelectThreads = 1024;

// Bits that order as the weights do: a larger weight has larger ones, -0 and 0 the same, a NaN the largest.
__device__ __forceinline__ uint32_t rank_of(float w) {
    if (w != w) return ~0u;
    const uint32_t u = as_u32(w + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// One workgroup per sequence and head.  The rank of the lightest token that is kept is found eight bits at a time from counts of those bits;
// then the tokens are walked in order, a kept one taking the next place.
__global__ __launch_bounds__(kSelectThreads) void spqt_kv_select_kernel(Cache c, int keep, int recent, int32_t *new_lengths, int32_t *kept) {
    __shared__ int counts[256];
    __shared__ int wave_sums[2][kSelectThreads / 64];
    __shared__ uint32_t found_prefix;
    __shared__ int found_rest;
    const int s = blockIdx.y, head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int length = length_of(c, s);
    const int late = recent < length ? recent : length, older = length - late;
    const int total = length < keep ? length : keep, pick = total - late;      // of the older ones; late <= total
    const int32_t *table = c.table + (size_t)s * c.max_blocks;
    auto rank_at = [&](int t) {
        const uint32_t page = (uint32_t)table[t / kBlock];
        return page < c.pages ? rank_of(c.weights[weight_at(c, page, head) + t % kBlock]) : ~0u;
    };

    // least: the rank of the lightest one picked; rest: how many of that rank are picked
    uint32_t least = 0;
    int rest = pick;
    if (pick > 0 && pick < older) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) counts[tid] = 0;
            __syncthreads();
            for (int t = tid; t < older; t += kSelectThreads) {
                const uint32_t rank = rank_at(t);
                if (shift == 24 || (rank ^ least) >> (shift + 8) == 0) atomicAdd(&counts[rank >> shift & 255], 1);
            }
            __syncthreads();
            if (tid < 64) {
                // lane l holds the four highest digits from 255 - 4 l down
                int mine[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += mine[i] = counts[255 - 4 * lane - i];
                int before = sum;
#pragma unroll
                for (int step = 1; step < 64; step *= 2) {
                    const int other = __shfl_up(before, step);
                    before += lane >= step ? other : 0;
                }
                before -= sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < rest && before + mine[i] >= rest) {
                        found_prefix = least | (uint32_t)(255 - 4 * lane - i) << shift;
                        found_rest = rest - before;
                    }
                    before += mine[i];
                }
            }
            __syncthreads();
            least = found_prefix;
            rest = found_rest;
        }
    } else if (pick <= 0) {
        least = ~0u;
        rest = 0;
    } else {
        rest = older;                                      // all of them: rank 0 is no number's
    }

    int32_t *out = kept + ((size_t)s * c.kv_heads + head) * (size_t)keep;
    int done = 0, ties = 0;                                // places taken and ties seen by the tokens before this stretch
    for (int t0 = 0; t0 < length; t0 += kSelectThreads) {
        const int t = t0 + tid;
        uint32_t rank = 0;
        if (t < older && pick > 0) rank = rank_at(t);
        const bool tie = t < older && rank == least && pick > 0;
        const uint64_t tied = __ballot(tie);
        if (lane == 0) wave_sums[0][wave] = __popcll(tied);
        __syncthreads();
        int ties_before = ties + (int)__popcll(tied & ((1ull << lane) - 1));
        for (int w = 0; w < kSelectThreads / 64; ++w) {
            ties_before += w < wave ? wave_sums[0][w] : 0;
            ties += wave_sums[0][w];
        }
        const bool mine = t < length && (t >= older || (pick > 0 && (rank > least || (tie && ties_before < rest))));
        const uint64_t all = __ballot(mine);
        if (lane == 0) wave_sums[1][wave] = __popcll(all);
        __syncthreads();
        int place = done + (int)__popcll(all & ((1ull << lane) - 1));
        for (int w = 0; w < kSelectThreads / 64; ++w) {
            place += w < wave ? wave_sums[1][w] : 0;
            done += wave_sums[1][w];
        }
        if (mine && place < keep) out[place] = t;
    }
    for (int i = total + tid; i < keep; i += kSelectThreads) out[i] = -1;
    if (head == 0 && tid == 0) new_lengths[s] = total;
}

// One workgroup per new page, head and side.
template <int D, bool BF16>
__global__ __launch_bounds__(kTileThreads) void spqt_kv_move_kernel(Cache c, int keep, const int32_t *new_table, int new_blocks, const int32_t *kept) {
    __shared__ Tile<D> tile;
    const int s = blockIdx.z, head = blockIdx.y >> 1, which = blockIdx.y & 1, block = blockIdx.x;
    const int length = length_of(c, s), total = length < keep ? length : keep;
    const int base = block * kBlock, to = total - base < kBlock ? total - base : kBlock;
    if (to <= 0) return;
    const uint32_t page = (uint32_t)new_table[(size_t)s * new_blocks + block];
    const bool there = page < c.pages;
    const int32_t *from = kept + ((size_t)s * c.kv_heads + head) * (size_t)keep + base;
    const int32_t *table = c.table + (size_t)s * c.max_blocks;
    uint32_t pair = 0;
    for (int p = (int)threadIdx.x; p < to * (D / 8); p += kTileThreads) {
        const int i = p / (D / 8), d = p % (D / 8) * 8, t = from[i];
        uint32_t old = (uint32_t)table[t / kBlock];
        const bool known = old < c.pages;
        if (!known) old = 0;
        const float scale = known ? c.scales[scale_at(c, old, head, which)] : __builtin_nanf("");
        const uint8_t *in = c.codes + codes_at(c, old, head, which);
        u32x4 x = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t byte = in[which ? (d + j) * kBlock + place_of(t % kBlock) : t % kBlock * D + d + j];
            x[j / 2] |= (uint32_t)value_of<BF16>(byte, scale) << (16 * (j % 2));
        }
        *reinterpret_cast<u32x4 *>(&tile.v[i][d]) = x;
        pair = larger_pair(larger_pair(pair, x.x), larger_pair(x.y, larger_pair(x.z, x.w)));
        if (to < kBlock) *reinterpret_cast<u32x4 *>(c.tail + (((size_t)s * c.kv_heads + head) * 2 + which) * (size_t)(kBlock * D) + p * 8) = x;
    }
    const float scale = scale_of<BF16>(largest_of(tile, pair));
    if (!there) return;
    store_tile<D, BF16>(c, tile, page, head, which, 0, to, scale);
    if (threadIdx.x == 0) c.scales[scale_at(c, page, head, which)] = scale;
    if (which == 0 && threadIdx.x < kBlock) {
        float w = 0.0f;
        if ((int)threadIdx.x < to) {
            const int t = from[threadIdx.x];
            const uint32_t old = (uint32_t)table[t / kBlock];
            w = old < c.pages ? c.weights[weight_at(c, old, head) + t % kBlock] : __builtin_nanf("");
        }
        c.weights[weight_at(c, page, head) + threadIdx.x] = w;
    }
}

}  // namespace

extern "C" int spqt_kv_evict(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept,
                             void *stream) {
    const int rc = check_cache(cache, true);
    if (rc != SPQT_OK) return rc;
    if (!cache->weights || !new_table || !new_lengths || !kept || new_lengths == cache->lengths || new_table == cache->table) return SPQT_EINVAL;
    if (keep < 1 || recent < 0 || recent > keep) return SPQT_EINVAL;
    if (keep > 1 << 30 || new_blocks < 1 || new_blocks > 1 << 24 || (int64_t)new_blocks * kBlock < keep) return SPQT_ESHAPE;
    if ((uintptr_t)new_table % 4 != 0 || (uintptr_t)new_lengths % 4 != 0 || (uintptr_t)kept % 4 != 0) return SPQT_EALIGN;
    hipLaunchKernelGGL(spqt_kv_select_kernel, dim3(cache->kv_heads, cache->sequences), dim3(kSelectThreads), 0, (hipStream_t)stream, view(*cache), keep, recent,
                       new_lengths, kept);
    const int most = cache->max_blocks < (keep + kBlock - 1) / kBlock ? cache->max_blocks : (keep + kBlock - 1) / kBlock;
    const dim3 grid(most, 2 * cache->kv_heads, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        hipLaunchKernelGGL((spqt_kv_move_kernel<decltype(dim)::value, decltype(bf16)::value>), grid, dim3(kTileThreads), 0, (hipStream_t)stream, view(*cache), keep,
                           new_table, new_blocks, kept);
    });
    return launched();
}
