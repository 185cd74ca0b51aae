// Attention of many rows over the cache: a workgroup takes kRows of a kv head's rows and goes through the blocks of tokens that they see; the codes of a
// block are made fp16 once, in shared memory, for all of them.
//
// With S^T = K Q^T a lane of v_mfma_f32_32x32x16_f16 has one row of Q and half of each 32 tokens, and what it has of P^T is an operand of
// O^T = V^T P^T if a line of V^T holds the tokens in that order: per 16 tokens the fours 0 and 2 for the lower lanes, 1 and 3 for the upper ones.
#include "kv_attend.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Rows of a wavefront: 64, as two operands that share every read of a block, where sums and queries leave the registers for it.
template <int D>
struct Shape {
    static constexpr int kTiles = D > 128 ? 1 : 2;
    static constexpr int kRows = kWaves * kTiles * 32;
    static constexpr int kKeyStride = D + 8, kValueStride = kBlock + 8;      // fp16 numbers; 16 lines are in 16 different sets of banks
};

template <int D>
struct Staged {                          // a block's codes on their way
    u32x4 keys[D / 64], values[(2 * D + kThreads - 1) / kThreads][2];

    __device__ __forceinline__ void fetch(const uint8_t *page) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) keys[i] = *reinterpret_cast<const u32x4 *>(page + (threadIdx.x + i * kThreads) * 16);
#pragma unroll
        for (int i = 0; i < (2 * D + kThreads - 1) / kThreads; ++i) {
            const int line = threadIdx.x + i * kThreads;      // element and half of the lanes
            if (2 * D % kThreads != 0 && line >= 2 * D) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                values[i][x] = *reinterpret_cast<const u32x4 *>(page + kBlock * D + (line / 2) * kBlock + (line % 2 + 2 * x) * 16);
        }
    }
    __device__ __forceinline__ void put_down(_Float16 *k, _Float16 *v) const {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const int at = (threadIdx.x + i * kThreads) * 16;
            _Float16 *to = k + at / D * Shape<D>::kKeyStride + at % D;
            *reinterpret_cast<f16x8 *>(to) = codes_f16(u32x2{keys[i].x, keys[i].y});
            *reinterpret_cast<f16x8 *>(to + 8) = codes_f16(u32x2{keys[i].z, keys[i].w});
        }
#pragma unroll
        for (int i = 0; i < (2 * D + kThreads - 1) / kThreads; ++i) {
            const int line = threadIdx.x + i * kThreads;
            if (2 * D % kThreads != 0 && line >= 2 * D) continue;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                *reinterpret_cast<f16x8 *>(v + line / 2 * Shape<D>::kValueStride + t * 16 + line % 2 * 8) = codes_f16(u32x2{values[i][0][t], values[i][1][t]});
        }
    }
};

__device__ __forceinline__ float halves_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(as_u32(v), as_u32(v), false, false);
    return __builtin_fmaxf(as_float(r[0]), as_float(r[1]));
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void spqt_kv_prompt_kernel(Cache c, Call a, int tiles) {
    typedef Shape<D> S;
    constexpr int kTiles = S::kTiles;
    __shared__ __attribute__((aligned(16))) _Float16 keys[2][kBlock * S::kKeyStride];
    __shared__ __attribute__((aligned(16))) _Float16 values[2][D * S::kValueStride];
    // heads first: workgroups of one head run on one XCD if there are eight; the rows that see most first
    const int s = blockIdx.z, head = blockIdx.x % c.kv_heads, tile = tiles - 1 - (int)(blockIdx.x / c.kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = lane & 31, half = lane >> 5;
    const int length = length_of(c, s), count = count_of(a.counts, s, a.rows), rows = a.rows * a.group;

    // the tokens that any, and that every row of the workgroup and of the wavefront sees
    const int r0 = tile * S::kRows;
    const Row first = row_of(a, r0, head, length, count);
    int last_live = r0 + S::kRows - 1 < count * a.group - 1 ? r0 + S::kRows - 1 : count * a.group - 1;
    const Row last = row_of(a, last_live < 0 ? 0 : last_live, head, length, count);
    const bool any = last_live >= r0 && last.high >= 0;
    const int begin = any ? block_of(first.high >= 0 ? first.low : 0) : 0, end = any ? block_of(last.high) + 1 : 0;

    Row row[kTiles];
    f16x8 q[kTiles][D / 16];
    float scale[kTiles], top[kTiles], total[kTiles], unit[kTiles];
    f32x16 acc[kTiles][D / 32];
    int full_low = 0, full_high = 0x7FFFFFFF;                 // every row of the wavefront sees these tokens
#pragma unroll
    for (int m = 0; m < kTiles; ++m) {
        const int r = r0 + (wave * kTiles + m) * 32 + column;
        row[m] = row_of(a, r, head, length, count);
        if (r >= rows) row[m].high = -1;
        const bool live = row[m].high >= 0;
        const uint16_t *from = a.q.data + s * a.q.sequence + row[m].i * a.q.row + row[m].head * a.q.head;
        u32x4 w[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) w[j] = live ? *reinterpret_cast<const u32x4 *>(from + 16 * j + 8 * half) : u32x4{0u, 0u, 0u, 0u};
        scale[m] = a.scale * kLog2e * queries_f16<BF16, D / 16>(w, q[m], 32);
        top[m] = kNone;
        total[m] = 0.0f;
        unit[m] = 1.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][i][e] = 0.0f;
        int low = row[m].low, high = row[m].high;
#pragma unroll
        for (int step = 1; step < 32; step *= 2) {
            const int l = __shfl_xor(low, step), h = __shfl_xor(high, step);
            low = l > low ? l : low;
            high = h < high ? h : high;
        }
        full_low = low > full_low ? low : full_low;
        full_high = high < full_high ? high : full_high;
    }
    full_low = __builtin_amdgcn_readfirstlane(full_low);
    full_high = __builtin_amdgcn_readfirstlane(full_high);

    const int32_t *table = c.table + (size_t)s * c.max_blocks;
    struct Page {
        const uint8_t *codes;
        float scale_k, scale_v;
    };
    auto page_of = [&](int block) {
        Page p;
        uint32_t page = (uint32_t)table[block];
        const bool there = page < c.pages;
        if (!there) page = 0;
        const float *scales = c.scales + scale_at(c, page, head, 0);
        p.codes = c.codes + codes_at(c, page, head, 0);
        p.scale_k = there ? scales[0] : __builtin_nanf("");
        p.scale_v = there ? scales[1] : __builtin_nanf("");
        return p;
    };

    auto attend = [&](int block, float scale_k, float scale_v, const _Float16 *k, const _Float16 *v, auto masked) {
        f32x16 p[kTiles][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const f16x8 x = *reinterpret_cast<const f16x8 *>(k + (32 * t + column) * S::kKeyStride + 16 * j + 8 * half);
#pragma unroll
                for (int m = 0; m < kTiles; ++m) {
                    if (j == 0) p[m][t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[m][j], f32x16{}, 0, 0, 0);
                    else p[m][t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[m][j], p[m][t], 0, 0, 0);
                }
            }
        }
        f16x8 lifted[kTiles][4];
#pragma unroll
        for (int m = 0; m < kTiles; ++m) {
            const float by = scale[m] * scale_k;
            if (decltype(masked)::value) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int token = block * kBlock + 32 * t + 8 * (e / 4) + 4 * half + e % 4;
                        if (!(token >= row[m].low && token <= row[m].high)) p[m][t][e] = kNone;
                    }
            }
            float most = p[m][0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = __builtin_fmaxf(most, p[m][t][e]);
            most = halves_max(most);
            const bool sees = !decltype(masked)::value || !(most == kNone);
            most = __builtin_fmaxf(top[m], sees ? most * by : kNone);
            const float from = most == kNone ? 0.0f : most;
            float shrink = __builtin_amdgcn_exp2f(top[m] - from);
            top[m] = most;
            total[m] *= shrink;
            if (sees) {
                shrink *= unit[m] / scale_v;
                unit[m] = scale_v;
            }
            const float lifted_from = from - 15.0f;
            float sum = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    f32x2 x;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(p[m][t][e + i], by, -lifted_from));
                        x[i] = decltype(masked)::value && p[m][t][e + i] == kNone ? 0.0f : y;
                        sum += x[i];
                    }
                    const f16x2 h = __builtin_convertvector(x, f16x2);
                    lifted[m][2 * t + e / 8][e % 8] = h[0];
                    lifted[m][2 * t + e / 8][e % 8 + 1] = h[1];
                }
            total[m] += sum * (1.0f / kLift);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[m][i] *= shrink;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f16x8 x = *reinterpret_cast<const f16x8 *>(v + (32 * i + column) * S::kValueStride + 16 * u + 8 * half);
#pragma unroll
                for (int m = 0; m < kTiles; ++m) acc[m][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, lifted[m][u], acc[m][i], 0, 0, 0);
            }
    };

    if (begin < end) {
        Staged<D> staged;
        Page now = page_of(begin), next = now;
        staged.fetch(now.codes);
        staged.put_down(keys[0], values[0]);
        if (begin + 1 < end) {
            next = page_of(begin + 1);
            staged.fetch(next.codes);
        }
        for (int block = begin; block < end; ++block) {
            const int b = (block - begin) & 1;
            __syncthreads();                                  // block's numbers are in place, and the other buffer is free
            if (block + 1 < end) staged.put_down(keys[b ^ 1], values[b ^ 1]);
            Page after = next;
            if (block + 2 < end) {
                after = page_of(block + 2);
                staged.fetch(after.codes);
            }
            if (block * kBlock >= full_low && block * kBlock + kBlock - 1 <= full_high) attend(block, now.scale_k, now.scale_v, keys[b], values[b], std::false_type());
            else attend(block, now.scale_k, now.scale_v, keys[b], values[b], std::true_type());
            now = next;
            next = after;
        }
    }

#pragma unroll
    for (int m = 0; m < kTiles; ++m) {
        const int r = r0 + (wave * kTiles + m) * 32 + column;
        Meeting sum;
        sum.top = top[m];
        const auto both = __builtin_amdgcn_permlane32_swap(as_u32(total[m]), as_u32(total[m]), false, false);
        sum.total = as_float(both[0]) + as_float(both[1]);
        if (r >= rows) continue;
        uint16_t *out = a.out.data + s * a.out.sequence + row[m].i * a.out.row + row[m].head * a.out.head + 4 * half;
        const float by = unit[m] * (1.0f / kLift) * sum.inverse();
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                uint16_t v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = narrow<BF16>(acc[m][i][e + x] * by);
                *reinterpret_cast<u32x2 *>(out + 32 * i + 2 * e) = u32x2{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16};
            }
        if (a.lse && half == 0) a.lse[((size_t)s * a.rows + row[m].i) * a.q_heads + row[m].head] = sum.lse();
    }
}

}  // namespace

namespace spqt {
namespace kv {

bool is_prompt(const Call &a, int) { return a.rows * a.group > 64; }

void launch_prompt(const spqt_kv_cache &cache, const Call &a, hipStream_t stream) {
    dispatch(cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        const int tiles = (a.rows * a.group + Shape<D>::kRows - 1) / Shape<D>::kRows;
        hipLaunchKernelGGL((spqt_kv_prompt_kernel<D, decltype(bf16)::value>), dim3((unsigned)tiles * cache.kv_heads, 1, cache.sequences), dim3(kThreads), 0, stream,
                           view(cache), a, tiles);
    });
}

}  // namespace kv
}  // namespace spqt
