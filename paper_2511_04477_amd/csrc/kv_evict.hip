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

constexpr int kSelectWaves = kSelectThreads / 64, kCopies = 16;
constexpr int kNearby = 34816;                            // ranks in shared memory, 136 KB

// One workgroup per sequence and head.  The rank of the lightest token that is kept is found eight bits at a time from counts of those bits, 16 copies of them
// for the lanes to keep out of each other's way; then every thread walks a stretch of tokens in order, a kept one taking the next place.
// What bounds it: one CU per sequence and head, for 5 passes over the tokens' ranks.  They stay in shared memory where there are at most 34816 of them.
__global__ __launch_bounds__(kSelectThreads) void spqt_kv_select_kernel(Cache c, int keep, int recent, int32_t *new_lengths, int32_t *kept) {
    extern __shared__ uint32_t ranks[];
    __shared__ int counts[256 * kCopies];
    __shared__ int wave_sums[2][kSelectWaves];
    __shared__ uint32_t found_prefix;
    __shared__ int found_rest;
    const int s = blockIdx.y, head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int length = length_of(c, s);
    const int late = recent < length ? recent : length, older = length - late;
    const int total = length < keep ? length : keep, pick = total - late;      // of the older ones; late <= total
    int32_t *out = kept + ((size_t)s * c.kv_heads + head) * (size_t)keep;
    if (head == 0 && tid == 0) new_lengths[s] = total;
    for (int i = total + tid; i < keep; i += kSelectThreads) out[i] = -1;
    if (pick <= 0 || pick == older) {                     // the last ones, or all
        for (int i = tid; i < total; i += kSelectThreads) out[i] = length - total + i;
        return;
    }

    const int32_t *table = c.table + (size_t)s * c.max_blocks;
    auto choose = [&](auto rank_at) {
    // least: the rank of the lightest one picked; rest: how many of that rank are picked
    uint32_t least = 0;
    int rest = pick;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256 * kCopies; i += kSelectThreads) counts[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int t = tid; t < older; t += kSelectThreads) {
            const uint32_t rank = rank_at(t);
            if (shift == 24 || (rank ^ least) >> (shift + 8) == 0) atomicAdd(&counts[(rank >> shift & 255) * kCopies + (lane & (kCopies - 1))], 1);
        }
        __syncthreads();
        if (tid < 256) {
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) sum += counts[tid * kCopies + (i + tid) % kCopies];
            counts[tid * kCopies] = sum;
        }
        __syncthreads();
        if (tid < 64) {
            // lane l holds the four highest digits from 255 - 4 l down
            int mine[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += mine[i] = counts[(255 - 4 * lane - i) * kCopies];
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

    // an odd stretch each, so that the lanes' ranks are in different banks
    const int stretch = ((older + kSelectThreads - 1) / kSelectThreads) | 1;
    const int begin = tid * stretch < older ? tid * stretch : older, end = begin + stretch < older ? begin + stretch : older;
    int heavier = 0, ties = 0;
    for (int t = begin; t < end; ++t) {
        const uint32_t rank = rank_at(t);
        heavier += rank > least;
        ties += rank == least;
    }
    auto before_me = [&](int mine, int *sums) {           // the sum of the threads before this one
        int upto = mine;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int other = __shfl_up(upto, step);
            upto += lane >= step ? other : 0;
        }
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int before = upto - mine;
        for (int w = 0; w < wave; ++w) before += sums[w];
        return before;
    };
    const int ties_before = before_me(ties, wave_sums[0]);
    int left = rest - ties_before;                        // of the ties that are picked
    left = left < 0 ? 0 : left;
    int place = before_me(heavier + (ties < left ? ties : left), wave_sums[1]);
    for (int t = begin; t < end; ++t) {
        const uint32_t rank = rank_at(t);
        const bool tie = rank == least && left > 0;
        left -= tie;
        if (rank > least || tie) out[place++] = t;
    }
    for (int i = tid; i < late; i += kSelectThreads) out[pick + i] = older + i;
    };
    if (older <= kNearby) {
        // a block per wavefront at a time, whose pages are looked up at once
        const int blocks = (older + kBlock - 1) / kBlock;
        for (int b0 = wave; b0 < blocks; b0 += 64 * kSelectWaves) {
            const int mine = b0 + lane * kSelectWaves;
            const uint32_t page = mine < blocks ? (uint32_t)table[mine] : 0u;
#pragma unroll 8
            for (int i = 0; i < 64; ++i) {
                const int b = b0 + i * kSelectWaves;
                if (b >= blocks) break;
                const uint32_t here = (uint32_t)__builtin_amdgcn_readlane((int)page, i);
                ranks[b * kBlock + lane] = here < c.pages ? rank_of(c.weights[weight_at(c, here, head) + lane]) : ~0u;
            }
        }
        __syncthreads();
        choose([&](int t) { return ranks[t]; });
    } else {
        choose([&](int t) {
            const uint32_t page = (uint32_t)table[t / kBlock];
            return page < c.pages ? rank_of(c.weights[weight_at(c, page, head) + t % kBlock]) : ~0u;
        });
    }
}

// One workgroup per new page, head and side.
template <int D, bool BF16>
__global__ __launch_bounds__(kTileThreads) void spqt_kv_move_kernel(Cache c, int keep, const int32_t *new_table, int new_blocks, const int32_t *kept) {
    __shared__ Tile<D> tile;
    __shared__ uint32_t pages[kBlock], tokens[kBlock];
    __shared__ float scales[kBlock];
    const int s = blockIdx.z, head = blockIdx.y >> 1, which = blockIdx.y & 1, block = blockIdx.x;
    const int length = length_of(c, s), total = length < keep ? length : keep;
    const int base = block * kBlock, to = total - base < kBlock ? total - base : kBlock;
    if (to <= 0) return;
    const uint32_t page = (uint32_t)new_table[(size_t)s * new_blocks + block];
    const bool there = page < c.pages;
    const int32_t *from = kept + ((size_t)s * c.kv_heads + head) * (size_t)keep + base;
    const int32_t *table = c.table + (size_t)s * c.max_blocks;
    if ((int)threadIdx.x < to) {
        const int t = from[threadIdx.x];
        uint32_t old = (uint32_t)table[t / kBlock];
        const bool known = old < c.pages;
        if (!known) old = 0;
        pages[threadIdx.x] = old;
        tokens[threadIdx.x] = (uint32_t)(t % kBlock);
        scales[threadIdx.x] = known ? c.scales[scale_at(c, old, head, which)] : __builtin_nanf("");
        if (which == 0 && there) c.weights[weight_at(c, page, head) + threadIdx.x] = known ? c.weights[weight_at(c, old, head) + t % kBlock] : __builtin_nanf("");
    } else if (threadIdx.x < kBlock) {
        pages[threadIdx.x] = tokens[threadIdx.x] = 0;
        scales[threadIdx.x] = 0.0f;
        if (which == 0 && there) c.weights[weight_at(c, page, head) + threadIdx.x] = 0.0f;
    }
    __syncthreads();
    uint32_t pair = 0;
    if (which == 0) {
        for (int p = (int)threadIdx.x; p < to * (D / 8); p += kTileThreads) {
            const int i = p / (D / 8), d = p % (D / 8) * 8;
            const u32x2 bytes = *reinterpret_cast<const u32x2 *>(c.codes + codes_at(c, pages[i], head, 0) + tokens[i] * D + d);
            u32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = values_of<BF16>(bytes[j / 2] >> (16 * (j % 2)) & 255, bytes[j / 2] >> (16 * (j % 2) + 8) & 255, scales[i]);
            tile.put(i, d, x);
            pair = larger_pair(larger_pair(pair, x.x), larger_pair(x.y, larger_pair(x.z, x.w)));
        }
    } else {
        // a token per lane: those that lie in one page have their bytes of an element in one line
        const int i = threadIdx.x & 63;
        const uint8_t *in = c.codes + codes_at(c, pages[i], head, 1) + place_of((int)tokens[i]);
        const float scale = scales[i];
#pragma unroll 8
        for (int d = (int)(threadIdx.x >> 6) * 2; d < D; d += kTileThreads / 64 * 2) {
            const uint32_t x = values_of<BF16>(in[d * kBlock], in[(d + 1) * kBlock], scale);
            *reinterpret_cast<uint32_t *>(&tile.v[i][d]) = x;
            if (i < to) pair = larger_pair(pair, x);
        }
    }
    const float scale = scale_of<BF16>(largest_of(tile, pair));
    if (!there) return;
    store_tile<D, BF16>(c, tile, page, head, which, 0, to, scale);
    if (threadIdx.x == 0) c.scales[scale_at(c, page, head, which)] = scale;
    if (to < kBlock) {
        uint16_t *tail = c.tail + (((size_t)s * c.kv_heads + head) * 2 + which) * (size_t)(kBlock * D);
        for (int p = (int)threadIdx.x; p < to * (D / 4); p += kTileThreads)
            *reinterpret_cast<u32x2 *>(tail + p * 4) = *reinterpret_cast<const u32x2 *>(&tile.v[p / (D / 4)][p % (D / 4) * 4]);
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
    // as many ranks in shared memory as the sequences' tables have room for
    const int64_t room = (int64_t)cache->max_blocks * kBlock;
    const size_t bytes = (size_t)(room < kNearby ? room : kNearby) * 4;
    hipLaunchKernelGGL(spqt_kv_select_kernel, dim3(cache->kv_heads, cache->sequences), dim3(kSelectThreads), bytes, (hipStream_t)stream, view(*cache), keep, recent,
                       new_lengths, kept);
    const int most = cache->max_blocks < (keep + kBlock - 1) / kBlock ? cache->max_blocks : (keep + kBlock - 1) / kBlock;
    const dim3 grid(most, 2 * cache->kv_heads, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        hipLaunchKernelGGL((spqt_kv_move_kernel<decltype(dim)::value, decltype(bf16)::value>), grid, dim3(kTileThreads), 0, (hipStream_t)stream, view(*cache), keep,
                           new_table, new_blocks, kept);
    });
    return launched();
}
