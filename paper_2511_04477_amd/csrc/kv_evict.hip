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
constexpr int kNearby = 32768;                            // ranks in shared memory, 128 KB

// One workgroup per sequence and head.  The rank of the lightest token that is kept is found eight bits at a time from counts of those bits, 16 copies of them
// for the lanes to keep out of each other's way; then every thread walks a stretch of tokens in order, a kept one taking the next place.
// What bounds it: one CU per sequence and head, for 6 passes over the tokens' ranks.  They stay in shared memory where there are at most 32768 of them (read
// once, 4 bytes a token): sequences of 27000 and 33001 tokens of 8 heads, 8192 kept, 24 us, and 17 more if every pass reads them from memory, as it does beyond; 2300 of 32 heads,
// 2048 kept, 10 us.
__global__ __launch_bounds__(kSelectThreads) void spqt_kv_select_kernel(Cache c, int keep, int recent, int32_t *new_lengths, int32_t *kept) {
    extern __shared__ __attribute__((aligned(16))) uint32_t ranks[];
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
    // four(t): the ranks of tokens t .. t + 3, 0 (no token's rank) for those from `older` on; t is a multiple of 4 below `upto`
    const int upto = (older + 4 * kSelectThreads - 1) / (4 * kSelectThreads) * (4 * kSelectThreads);
    auto choose = [&](auto four) {
        // least: the rank of the lightest one picked; rest: how many of that rank are picked
        uint32_t least = 0;
        int rest = pick;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256 * kCopies; i += kSelectThreads) counts[i] = 0;
            __syncthreads();
            int *mine = counts + (lane & (kCopies - 1));
#pragma unroll 2
            for (int t = 4 * tid; t < upto; t += 4 * kSelectThreads) {
                const u32x4 rank = four(t);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (shift == 24 || (rank[i] ^ least) >> (shift + 8) == 0) atomicAdd(mine + (rank[i] >> shift & 255) * kCopies, 1);
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
                int here[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += here[i] = counts[(255 - 4 * lane - i) * kCopies];
                int before = (int)sum_upto((uint32_t)sum) - sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < rest && before + here[i] >= rest) {
                        found_prefix = least | (uint32_t)(255 - 4 * lane - i) << shift;
                        found_rest = rest - before;
                    }
                    before += here[i];
                }
            }
            __syncthreads();
            least = found_prefix;
            rest = found_rest;
        }

        // every wavefront walks its stretch, 256 tokens at a time, once to count and once to write
        const int steps = upto / 256, begin = steps * wave / kSelectWaves * 256, end = steps * (wave + 1) / kSelectWaves * 256;
        int heavier = 0, ties = 0;
#pragma unroll 2
        for (int t = begin + 4 * lane; t < end; t += 256) {
            const u32x4 rank = four(t);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                heavier += rank[i] > least;
                ties += rank[i] == least;
            }
        }
        heavier = (int)lane_of(sum_upto((uint32_t)heavier), 63);
        ties = (int)lane_of(sum_upto((uint32_t)ties), 63);
        if (lane == 0) {
            wave_sums[0][wave] = heavier;
            wave_sums[1][wave] = ties;
        }
        __syncthreads();
        int place = 0, left = rest;                       // of the ties that are picked
        for (int w = 0; w < wave; ++w) {
            const int here = left < wave_sums[1][w] ? left : wave_sums[1][w];
            place += wave_sums[0][w] + here;
            left -= here;
        }
        for (int t = begin + 4 * lane; t < end; t += 256) {
            const u32x4 rank = four(t);
            bool picked[4];
            int mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) picked[i] = rank[i] > least;
            if (left > 0 && __ballot(rank[0] == least || rank[1] == least || rank[2] == least || rank[3] == least)) {
                int tied = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) tied += rank[i] == least;
                const int all = (int)sum_upto((uint32_t)tied);
                int before = all - tied;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (rank[i] == least) picked[i] = before++ < left;
                const int here = (int)lane_of((uint32_t)all, 63);
                left -= left < here ? left : here;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) mine += picked[i];
            const int all = (int)sum_upto((uint32_t)mine);
            int *to = out + place + all - mine;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (picked[i]) *to++ = t + i;
            place += (int)lane_of((uint32_t)all, 63);
        }
        for (int i = tid; i < late; i += kSelectThreads) out[pick + i] = older + i;
    };
    if (older <= kNearby) {
        // A wavefront's blocks, whose pages are looked up at once, and all their weights are on their way together.  Up to 8192 tokens a copy
        // of the code has no steps for more: 2300 tokens of 32 heads 34.2 us for 35.3 (eviction and read), 4000 of 8 heads 22.2 for 23.3; from 9000 on 65.9 for 65.8.
        const int blocks = (older + kBlock - 1) / kBlock, mine = wave + lane * kSelectWaves;
        const uint32_t page = mine < blocks ? (uint32_t)table[mine] : ~0u;
        auto fetch = [&](auto most) {
            constexpr int kMost = decltype(most)::value;
            float w[kMost];
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const uint32_t here = lane_of(page, i);
                if (here < c.pages) w[i] = c.weights[weight_at(c, here, head) + lane];
            }
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const uint32_t here = lane_of(page, i);
                const int b = wave + i * kSelectWaves, t = b * kBlock + lane;
                if (b * kBlock < upto) ranks[t] = t >= older ? 0u : (here < c.pages ? rank_of(w[i]) : ~0u);
            }
        };
        constexpr int kAll = kNearby / kBlock / kSelectWaves, kFew = 8;
        static_assert(kAll <= 64 && kAll * kBlock * kSelectWaves == kNearby && kNearby % (4 * kSelectThreads) == 0, "blocks of a wavefront");
        if (upto <= kFew * kBlock * kSelectWaves) fetch(std::integral_constant<int, kFew>());
        else fetch(std::integral_constant<int, kAll>());
        __syncthreads();
        choose([&](int t) { return *reinterpret_cast<const u32x4 *>(ranks + t); });
    } else {
        choose([&](int t) {
            u32x4 rank = {0u, 0u, 0u, 0u};
            if (t < older) {
                const uint32_t page = (uint32_t)table[t / kBlock];
                if (page < c.pages) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(c.weights + weight_at(c, page, head) + t % kBlock);
                    rank = u32x4{rank_of(w.x), rank_of(w.y), rank_of(w.z), rank_of(w.w)};
                } else {
                    rank = ~rank;
                }
#pragma unroll
                for (int i = 1; i < 4; ++i) rank[i] = t + i < older ? rank[i] : 0u;
            }
            return rank;
        });
    }
}

// Kept tokens quantized as a new block.  By way of 16 bits: x = code * scale as spqt_kv_read gives it, then as in the append.  EXACT: from code * scale itself, 20 bits at most; a block whose
// tokens all stay then keeps its scale and codes, since 127 * scale asks for just that scale, while 127 * scale rounded to 11 bits may ask for the next one.  (Either takes the same time: selection and move of the two sequences below 55.4 and 54.9 us, of the 32 heads 24.2 and 24.0.)
// One workgroup per new page, head and side.  Keys are whole lines of a token; values, a byte of each of D lines, are read a token per lane, since tokens that are kept of one page
// then share lines.
// What bounds it: those lines.  27000 and 33001 tokens of 8 heads of 128, 8192 kept of each, 37 us for the 68 MB of the codes that are kept and written; where nearly all are kept
// (2048 of 2300, 32 heads) 15.7 us for 34 MB.
template <int D, bool BF16, bool EXACT>
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
    uint32_t pair = 0;                                    // the largest magnitudes of a pair of numbers, or the largest code * scale
    auto larger = [&](int token, uint32_t code) {
        const float x = (float)code * scales[token];
        pair = as_u32(x) > pair ? as_u32(x) : pair;
    };
    auto magnitude = [](uint32_t byte) { return byte > 128 ? byte - 128 : 128 - byte; };
    if (which == 0) {
        u32x2 bytes[D / 32];
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            const int p = (int)threadIdx.x + n * kTileThreads, i = p / (D / 8);
            bytes[n] = *reinterpret_cast<const u32x2 *>(c.codes + codes_at(c, pages[i], head, 0) + tokens[i] * D + p % (D / 8) * 8);
        }
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            const int p = (int)threadIdx.x + n * kTileThreads, i = p / (D / 8);
            u32x4 x;
            uint32_t most = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t first = bytes[n][j / 2] >> (16 * (j % 2)) & 255, second = bytes[n][j / 2] >> (16 * (j % 2) + 8) & 255;
                x[j] = EXACT ? first | second << 16 : values_of<BF16>(first, second, scales[i]);
                most = magnitude(first) > most ? magnitude(first) : most;
                most = magnitude(second) > most ? magnitude(second) : most;
            }
            tile.put(i, p % (D / 8) * 8, x);
            if (EXACT && i < to) larger(i, most);
            if (!EXACT && i < to) pair = larger_pair(larger_pair(pair, x.x), larger_pair(x.y, larger_pair(x.z, x.w)));
        }
    } else {
        // a token per lane: those that lie in one page have their bytes of an element in one line
        const int i = threadIdx.x & 63;
        const uint8_t *in = c.codes + codes_at(c, pages[i], head, 1) + place_of((int)tokens[i]);
        const float scale = scales[i];
        uint32_t most = 0;
#pragma unroll 8
        for (int d = (int)(threadIdx.x >> 6) * 2; d < D; d += kTileThreads / 64 * 2) {
            const uint32_t first = in[d * kBlock], second = in[(d + 1) * kBlock];
            const uint32_t x = EXACT ? first | second << 16 : values_of<BF16>(first, second, scale);
            *reinterpret_cast<uint32_t *>(&tile.v[i][d]) = x;
            if (EXACT) {
                most = magnitude(first) > most ? magnitude(first) : most;
                most = magnitude(second) > most ? magnitude(second) : most;
            } else if (i < to) {
                pair = larger_pair(pair, x);
            }
        }
        if (EXACT && i < to) larger(i, most);
    }
    if (EXACT) {
        const uint32_t largest = largest_number(tile, pair);
        const float scale = largest >= 0x7F800000u ? __builtin_nanf("") : scale_for(as_float(largest));
        if (!there) return;
        // old scale / new scale; more than 128 only where the token's codes are all 0
        if (threadIdx.x < kBlock) scales[threadIdx.x] = __builtin_fminf(scales[threadIdx.x] / scale, 128.0f);
        __syncthreads();
        // code times that to the nearest integer, in one rounding
        auto code = [&](uint32_t pair, int upper, int t) {
            return as_u32(__builtin_fmaf((float)((int)(upper ? pair >> 16 : pair & 0xFFFFu) - 128), scales[t], 12582912.0f + 128.0f));
        };
        store_codes(c, tile, page, head, which, 0, to, scale, code);
        if (threadIdx.x == 0) c.scales[scale_at(c, page, head, which)] = scale;
        if (to == kBlock) return;
        uint16_t *tail = c.tail + (((size_t)s * c.kv_heads + head) * 2 + which) * (size_t)(kBlock * D);
        for (int p = (int)threadIdx.x; p < to * (D / 2); p += kTileThreads) {
            const int t = p / (D / 2), d = p % (D / 2) * 2;
            const uint32_t pair = *reinterpret_cast<const uint32_t *>(&tile.v[t][d]);
            *reinterpret_cast<uint32_t *>(tail + p * 2) = values_of<BF16>(code(pair, 0, t) & 255, code(pair, 1, t) & 255, scale);
        }
        return;
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

static int evict(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept, void *stream, bool exact) {
    const int rc = check_cache(cache, true);
    if (rc != SPQT_OK) return rc;
    if (!cache->weights || !new_table || !new_lengths || !kept || new_lengths == cache->lengths || new_table == cache->table) return SPQT_EINVAL;
    if (keep < 1 || recent < 0 || recent > keep) return SPQT_EINVAL;
    if (keep > 1 << 30 || new_blocks < 1 || new_blocks > 1 << 24 || (int64_t)new_blocks * kBlock < keep) return SPQT_ESHAPE;
    if ((uintptr_t)new_table % 4 != 0 || (uintptr_t)new_lengths % 4 != 0 || (uintptr_t)kept % 4 != 0) return SPQT_EALIGN;
    // as many ranks in shared memory as the sequences' tables have room for
    const int64_t room = ((int64_t)cache->max_blocks * kBlock + 4 * kSelectThreads - 1) / (4 * kSelectThreads) * (4 * kSelectThreads);
    const size_t bytes = (size_t)(room < kNearby ? room : kNearby) * 4;
    hipLaunchKernelGGL(spqt_kv_select_kernel, dim3(cache->kv_heads, cache->sequences), dim3(kSelectThreads), bytes, (hipStream_t)stream, view(*cache), keep, recent,
                       new_lengths, kept);
    const int most = cache->max_blocks < (keep + kBlock - 1) / kBlock ? cache->max_blocks : (keep + kBlock - 1) / kBlock;
    const dim3 grid(most, 2 * cache->kv_heads, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), 0, (hipStream_t)stream, view(*cache), keep, new_table, new_blocks, kept);
        };
        if (exact) launch(spqt_kv_move_kernel<decltype(dim)::value, decltype(bf16)::value, true>);
        else launch(spqt_kv_move_kernel<decltype(dim)::value, decltype(bf16)::value, false>);
    });
    return launched();
}

extern "C" int spqt_kv_evict(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept,
                             void *stream) {
    return evict(cache, keep, recent, new_table, new_blocks, new_lengths, kept, stream, false);
}

extern "C" int spqt_kv_evict_exact(const spqt_kv_cache *cache, int keep, int recent, const int32_t *new_table, int new_blocks, int32_t *new_lengths, int32_t *kept,
                                   void *stream) {
    return evict(cache, keep, recent, new_table, new_blocks, new_lengths, kept, stream, true);
}
