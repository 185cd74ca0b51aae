// What every cached token weighed in a call: the sum of the probabilities that the rows gave it, whose sums (lse) are known.  The scores are worked out again:
// they would take as much memory as the rows see tokens, and keys are half of what the attention read.
#include "kv_attend.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

// A few rows: a wavefront per block, which goes over all rows.
// What bounds it: the keys, 29300 tokens of 8 heads of 128 (30 MB, from the cache behind memory) 12.6 us = 2.4 TB/s: a start, one chain of loads and a tail per block.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void spqt_kv_weigh_few_kernel(Cache c, Call a) {
    const int s = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, column = lane & 15, quarter = lane >> 4;
    const int block = blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int length = length_of(c, s), count = count_of(a.counts, s, a.rows);
    if (block * kBlock >= length) return;
    const uint32_t page = (uint32_t)c.table[(size_t)s * c.max_blocks + block];
    if (page >= c.pages) return;
    const float scale_k = c.scales[scale_at(c, page, head, 0)];
    const uint8_t *keys = c.codes + codes_at(c, page, head, 0);
    u32x4 k[4][D / 64];
#pragma unroll
    for (int t = 0; t < 4; ++t) load_keys<D>(k[t], keys, t, lane);
    f32x4 sum[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) sum[t] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r0 = 0; r0 < count * a.group; r0 += 16) {
        const int r = r0 + column;
        const bool inside = r < count * a.group;
        Row row = row_of(a, r, head, length, count);
        if (!inside) row.high = -1;
        if (rows_max(row.high) < block * kBlock) continue;
        u32x4 raw[D / 32];
        f16x8 q[D / 32];
        load_queries<D>(raw, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, row.high >= 0, lane);
        const float positive = positive_scale(a.scale, raw), back = queries_f16<BF16>(raw, q, 16);
        const float scale = positive * back * kLog2e * scale_k;
        const float whole = row.high >= 0 ? a.lse[((size_t)s * a.rows + row.i) * a.q_heads + row.head] * kLog2e : 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const f32x4 p = scores_of<D>(k[t], q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int token = block * kBlock + 16 * t + 4 * quarter + e;
                sum[t][e] += token >= row.low && token <= row.high ? __builtin_amdgcn_exp2f(p[e] * scale - whole) : 0.0f;
            }
        }
    }
    // lane `column` of a token's 16 takes the column-th of its quarter's tokens
    float mine = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = rows_sum(sum[t][e]);
            mine = column == 4 * t + e ? x : mine;
        }
    const int at = 16 * (column / 4) + 4 * quarter + column % 4;
    float *weight = c.weights + weight_at(c, page, head) + at;
    if (block * kBlock + at < length) *weight = a.decay == 0.0f ? mine : __builtin_fmaf(a.decay, *weight, mine);
}

// Many rows: a workgroup per block, whose wavefronts hold its keys as 16-bit numbers of the queries' type (a code is exact in either) and take every eighth (fourth)
// 32 of the rows that see it.  With S^T = K Q^T a lane has one row and half of each 32 tokens; its tokens' sums meet at the end.
// What bounds it: 32 exponentials and as many multiply-adds and additions a lane for 16 matrix instructions: 4001 rows of 32 / 8 heads from an empty cache 116 us (vector units busy for 0.60 of the time, matrix units for 0.30), 1024 rows of 64 / 8
// heads over 8192 tokens 196 us.
constexpr int many_threads(int dim) { return dim > 128 ? 256 : 512; }

template <int D, bool BF16>
__global__ __launch_bounds__(many_threads(D)) void spqt_kv_weigh_many_kernel(Cache c, Call a, int sequences) {
    constexpr int kManyWaves = many_threads(D) / 64;
    constexpr int kLine = D + 8;                              // 16-bit numbers; 16 lines are in 16 different sets of banks
    __shared__ float sums[kManyWaves][kBlock];
    __shared__ __attribute__((aligned(16))) uint16_t queries[kManyWaves][32 * kLine];
    const int s = blockIdx.z % sequences, head = blockIdx.x;                 // the blocks that most rows see first
    const int block = (int)(blockIdx.z / sequences * gridDim.y + blockIdx.y);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = lane & 31, half = lane >> 5;
    const int length = length_of(c, s), count = count_of(a.counts, s, a.rows), base = block * kBlock;
    if (base >= length) return;
    const uint32_t page = (uint32_t)c.table[(size_t)s * c.max_blocks + block];
    if (page >= c.pages) return;
    const float scale_k = c.scales[scale_at(c, page, head, 0)];
    const uint8_t *keys = c.codes + codes_at(c, page, head, 0);
    u32x4 k[2][D / 16];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const u32x2 codes = *reinterpret_cast<const u32x2 *>(keys + (32 * t + column) * D + 16 * j + 8 * half);
            const f16x8 x = codes_f16(codes);
            if (BF16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) k[t][j][i] = narrow2<true>((float)x[2 * i], (float)x[2 * i + 1]);
            } else {
                k[t][j] = __builtin_bit_cast(u32x4, x);
            }
        }
    // rows of the call that may see the block: from the position of its first token on, and no further than the window
    const int row0 = length - count;
    int first = base - row0, last = count - 1;                // (of the call; at or before the last one at position length - 1)
    first = first < 0 ? 0 : first;
    if (a.window > 0 && (int64_t)base + kBlock - 2 + a.window - row0 < last) last = base + kBlock - 2 + a.window - row0;
    const float by = a.scale * kLog2e * scale_k;
    f32x16 sum[2] = {f32x16{}, f32x16{}};

    // 32 rows from r0 = i0 * group + g0 on: where row r0 + t is, for small t
    const float inverse = 1.0f / (float)a.group;
    auto place = [&](int t, int g0, int &i, int &g) {
        i = (int)(((float)(t + g0) + 0.5f) * inverse);
        g = t + g0 - i * a.group;
    };
    const int end = (last + 1) * a.group, step = kManyWaves * 32;
    // A row's 16 lanes load it together, which the matrix instructions' order does not; they get it from the wavefront's part of shared memory.  Where the
    // pieces of 32 rows lie from the first one's on is the same for all of them if a step is whole positions, and is worked out once.
    u32x4 staged[D / 16];
    int64_t offsets[D / 16];
    float whole;
    Row row;
    auto find_pieces = [&](int g0, int most) {                // `most`: positions behind the last one are not followed
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            const int p = n * 64 + lane;
            int i, g;
            place(p / (D / 8), g0, i, g);
            offsets[n] = (i < most ? i : most) * a.q.row + g * a.q.head + p % (D / 8) * 8;
        }
    };
    auto fetch = [&](int r0) {
        const int i0 = r0 / a.group, g0 = r0 % a.group;       // (uniform)
        if (step % a.group != 0 || r0 + 32 > end) find_pieces(g0, last - i0);
        const uint16_t *from = a.q.data + s * a.q.sequence + (int64_t)head * a.group * a.q.head + i0 * a.q.row;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) staged[n] = *reinterpret_cast<const u32x4 *>(from + offsets[n]);
        int i, g;
        place(column, g0, i, g);
        i += i0;
        const int at = row0 + i;
        const bool live = i <= last && at >= 0;
        row.high = live ? at : -1;
        row.low = live && a.window > 0 && at - a.window + 1 > 0 ? at - a.window + 1 : 0;
        whole = a.lse[((size_t)s * a.rows + (i < last ? i : last)) * a.q_heads + head * a.group + g];
    };
    uint16_t *mine = queries[wave];
    int r0 = __builtin_amdgcn_readfirstlane(first * a.group + wave * 32);
    if (r0 < end) {
        find_pieces(r0 % a.group, last - r0 / a.group);
        fetch(r0);
    }
    for (; r0 < end; r0 += step) {
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            const int p = n * 64 + lane;
            *reinterpret_cast<u32x4 *>(mine + p / (D / 8) * kLine + p % (D / 8) * 8) = staged[n];
        }
        const Row now = row;
        const float now_whole = whole * kLog2e;
        if (r0 + step < end) fetch(r0 + step);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        f32x16 p[2];
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const f32x16 before = j == 0 ? f32x16{} : p[t];
                const u32x4 q = *reinterpret_cast<const u32x4 *>(mine + column * kLine + 16 * j + 8 * half);
                if (BF16) p[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[t][j]), __builtin_bit_cast(bf16x8, q), before, 0, 0, 0);
                else p[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, k[t][j]), __builtin_bit_cast(f16x8, q), before, 0, 0, 0);
            }
        const bool all = !__ballot(now.low > base || now.high < base + kBlock - 1);
        if (all) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[t][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(p[t][e], by, -now_whole));
        } else {
            asm volatile("");                                 // a branch: few blocks of a row are masked
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int token = base + 32 * t + 8 * (e / 4) + 4 * half + e % 4;
                    sum[t][e] += token >= now.low && token <= now.high ? __builtin_amdgcn_exp2f(__builtin_fmaf(p[t][e], by, -now_whole)) : 0.0f;
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");       // the reads are done before the next rows are put there
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float x = rows_sum(sum[t][e]);                    // of the 16 lanes, then of both of the half's
            const auto both = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
            x = as_float(both[0]) + as_float(both[1]);
            if (column == 0) sums[wave][32 * t + 8 * (e / 4) + 4 * half + e % 4] = x;
        }
    __syncthreads();
    if (threadIdx.x >= kBlock || base + (int)threadIdx.x >= length) return;
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kManyWaves; ++w) x += sums[w][threadIdx.x];
    float *weight = c.weights + weight_at(c, page, head) + threadIdx.x;
    *weight = a.decay == 0.0f ? x : __builtin_fmaf(a.decay, *weight, x);
}

}  // namespace

namespace spqt {
namespace kv {

void launch_weigh(const spqt_kv_cache &cache, const Call &a, hipStream_t stream) {
    dispatch(cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        constexpr bool B = decltype(bf16)::value;
        const int y = cache.max_blocks < 32768 ? cache.max_blocks : 32768;
        if ((int64_t)a.rows * a.group > kFewRows)
            hipLaunchKernelGGL((spqt_kv_weigh_many_kernel<D, B>), dim3(cache.kv_heads, y, (unsigned)cache.sequences * ((cache.max_blocks + y - 1) / y)),
                               dim3(many_threads(D)), 0, stream, view(cache), a, cache.sequences);
        else
            hipLaunchKernelGGL((spqt_kv_weigh_few_kernel<D, B>), dim3((cache.max_blocks + kWaves - 1) / kWaves, cache.kv_heads, cache.sequences), dim3(kThreads), 0, stream,
                               view(cache), a);
    });
}

}  // namespace kv
}  // namespace spqt
