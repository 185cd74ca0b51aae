// spqt_kv_attention: attention of some rows over the cache, softmax statistics of one pass (running maximum and sum), and what
// every cached token weighed in it.
//
// The rows that share a kv head - row i of the call and query head g of the head's group - are numbered r = i * group + g and taken 16 at a
// time.  With S^T = K Q^T a lane of v_mfma_f32_16x16x32_f16 has ONE row of Q and four tokens of each 16, and what it has of P^T is what it
// needs as an operand of O^T = V^T P^T, given the order in which a page holds the values (place_of): probabilities never leave their lane.
// Codes are exact in fp16, so the products are those of the 16-bit queries with the codes; the scale of a block goes into its scores and
// into its probabilities.
#include "kv_common.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();
// Probabilities go to the matrix instructions as two fp16 numbers, 22 bits in all, times 2^15: fp16's smallest number is 2^-39 of the largest one.
constexpr float kLift = 0x1p15f;

struct Call {
    Rows q, out;
    float *lse;
    const int32_t *counts;
    int rows, q_heads, group, window;
    float scale, decay;
};

// A lane's row: its place in the call, and the tokens low .. high that it sees (none if high < low).
struct Row {
    int i, head;
    int low, high;
};
__device__ __forceinline__ Row row_of(const Call &a, int r, int head, int length, int count) {
    Row w;
    w.i = r / a.group;
    w.head = head * a.group + r % a.group;
    const int at = length - count + w.i;
    const bool live = w.i < count && at >= 0 && at < length;
    w.high = live ? at : -1;
    w.low = live ? (a.window > 0 && at - a.window + 1 > 0 ? at - a.window + 1 : 0) : 0;
    return w;
}

__device__ __forceinline__ int lanes_max(int v) {            // over the 16 rows
#pragma unroll
    for (int step = 1; step < 16; step *= 2) {
        const int o = __shfl_xor(v, step);
        v = o > v ? o : v;
    }
    return v;
}
__device__ __forceinline__ float columns_max(float v) {      // over the four lanes of a row
    v = __builtin_fmaxf(v, __shfl_xor(v, 16));
    return __builtin_fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float columns_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// A row of Q as an operand, 32 elements a step: step j of a lane are elements 64 (j / 2) + 16 (lane / 16) + 8 (j % 2) on, as in load_keys.
// bf16 rows are scaled by a power of two to have their largest element in 2^14 .. 2^15, where fp16 holds them (exactly, down to
// 2^-30 of the largest); the factor that undoes it is returned.
template <int D, bool BF16>
__device__ __forceinline__ float load_queries(f16x8 (&q)[D / 32], const uint16_t *row, bool live, int lane) {
    u32x4 w[D / 32];
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
        w[j] = live ? *reinterpret_cast<const u32x4 *>(row + 64 * (j / 2) + 16 * (lane / 16) + 8 * (j % 2)) : u32x4{0u, 0u, 0u, 0u};
    if (!BF16) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) q[j] = __builtin_bit_cast(f16x8, w[j]);
        return 1.0f;
    }
    uint32_t largest = 0;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t a = w[j][e] & 0x7FFFu, b = w[j][e] >> 16 & 0x7FFFu;
            largest = largest > a ? largest : a;
            largest = largest > b ? largest : b;
        }
    for (int step = 16; step < 64; step *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)largest, step);
        largest = o > largest ? o : largest;
    }
    // exponent field of the largest, kept where 2^(141 - e) and its inverse are numbers; an infinity or a NaN stays what it is
    const int e = clamped((int)(largest >> 7), 20, 254);
    const float up = as_float((uint32_t)(268 - e) << 23), down = as_float((uint32_t)(e - 14) << 23);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int x = 0; x < 8; ++x) q[j][x] = (_Float16)(as_float(x % 2 ? w[j][x / 2] & 0xFFFF0000u : w[j][x / 2] << 16) * up);
    return down;
}

// 16 tokens' keys as an operand.
template <int D>
__device__ __forceinline__ void load_keys(u32x4 (&k)[D / 64], const uint8_t *page, int tile, int lane) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) k[j] = *reinterpret_cast<const u32x4 *>(page + (16 * tile + lane % 16) * D + 64 * j + 16 * (lane / 16));
}

template <int D>
__device__ __forceinline__ f32x4 scores_of(const u32x4 (&k)[D / 64], const f16x8 (&q)[D / 32]) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const u32x2 half = {k[j / 2][2 * (j % 2)], k[j / 2][2 * (j % 2) + 1]};
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(half), q[j], s, 0, 0, 0);
    }
    return s;
}

// One workgroup per 16 rows, kv head and sequence; its wavefronts take every fourth block of tokens, and their sums are joined at the end.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void spqt_kv_attend_kernel(Cache c, Call a) {
    __shared__ float sums[kWaves][16][D + 4];
    __shared__ float stats[kWaves][2][16];
    const int s = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = lane & 15, quarter = lane >> 4;
    const int length = length_of(c, s), count = count_of(a.counts, s, a.rows);
    const int r = blockIdx.x * 16 + column;
    const bool inside = r < a.rows * a.group;
    Row row = row_of(a, r, head, length, count);
    if (!inside) row.high = -1;
    f16x8 q[D / 32];
    const float back = load_queries<D, BF16>(q, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, inside && row.high >= 0, lane);
    const float scale = a.scale * back * kLog2e;

    float top = kNone, total = 0.0f, unit = 0x1p-120f;       // running maximum and sum of a row; the scale that acc is in
    f32x4 acc[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int high = lanes_max(row.high), low = high < 0 ? 0 : -lanes_max(row.high < 0 ? -0x7FFFFFFF : -row.low);
    for (int block = block_of(low) + wave; high >= 0 && block <= block_of(high); block += kWaves) {
        uint32_t page = (uint32_t)c.table[(size_t)s * c.max_blocks + block];
        const bool there = page < c.pages;
        if (!there) page = 0;
        const float scale_k = there ? c.scales[scale_at(c, page, head, 0)] : __builtin_nanf(""), scale_v = there ? c.scales[scale_at(c, page, head, 1)] : __builtin_nanf("");
        const uint8_t *keys = c.codes + codes_at(c, page, head, 0), *values = c.codes + codes_at(c, page, head, 1);
        f32x4 p[4];
        float most = top;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u32x4 k[D / 64];
            load_keys<D>(k, keys, t, lane);
            p[t] = scores_of<D>(k, q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int token = block * kBlock + 16 * t + 4 * quarter + e;
                p[t][e] = token >= row.low && token <= row.high ? p[t][e] * (scale * scale_k) : kNone;
                most = __builtin_fmaxf(most, p[t][e]);
            }
        }
        most = columns_max(most);
        const float from = most == kNone ? 0.0f : most;      // nothing seen yet: 2^(-inf - 0)
        float shrink = __builtin_amdgcn_exp2f(top - from);
        total *= shrink;
        top = most;
        if (scale_v > unit) {
            shrink *= unit / scale_v;
            unit = scale_v;
        }
        const float ratio = scale_v / unit * kLift;
        f16x8 lifted[2], rest[2];                            // a probability in units of `unit`
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool seen = !(p[t][e] == kNone);       // a NaN is one
                const float x = __builtin_amdgcn_exp2f(p[t][e] - from);
                total += x;
                const float y = seen ? x * ratio : 0.0f;
                const _Float16 h = (_Float16)y;
                lifted[t / 2][4 * (t % 2) + e] = h;
                rest[t / 2][4 * (t % 2) + e] = (_Float16)(y - (float)h);
            }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(values + (16 * i + column) * kBlock + 16 * quarter);
            acc[i] *= shrink;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const f16x8 codes = codes_f16(u32x2{v[2 * u], v[2 * u + 1]});
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, lifted[u], acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, rest[u], acc[i], 0, 0, 0);
            }
        }
    }
    total = columns_sum(total);

    const float drop = unit * (1.0f / kLift);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&sums[wave][column][16 * i + 4 * quarter]) = acc[i] * drop;
    if (quarter == 0) {
        stats[wave][0][column] = top;
        stats[wave][1][column] = total;
    }
    __syncthreads();
    const int mine = threadIdx.x / 16, r_out = blockIdx.x * 16 + mine, d0 = threadIdx.x % 16 * (D / 16);
    if (r_out >= a.rows * a.group) return;
    float all = kNone, whole = 0.0f, part[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all = __builtin_fmaxf(all, stats[w][0][mine]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        part[w] = __builtin_amdgcn_exp2f(stats[w][0][mine] - (all == kNone ? 0.0f : all));
        whole += part[w] * stats[w][1][mine];
    }
    const float inverse = whole == 0.0f ? 0.0f : 1.0f / whole;
    const int i_out = r_out / a.group, head_out = head * a.group + r_out % a.group;
    uint16_t *out = a.out.data + s * a.out.sequence + i_out * a.out.row + head_out * a.out.head + d0;
#pragma unroll
    for (int d = 0; d < D / 16; d += 4) {
        uint16_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) x += part[w] * sums[w][mine][d0 + d + e];
            v[e] = narrow<BF16>(x * inverse);
        }
        *reinterpret_cast<u32x2 *>(out + d) = u32x2{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16};
    }
    if (a.lse && threadIdx.x % 16 == 0)
        a.lse[((size_t)s * a.rows + i_out) * a.q_heads + head_out] = whole == 0.0f ? kNone : (all == kNone ? 0.0f : all) * kLn2 + __builtin_logf(whole);
}

// What the tokens weighed: a wavefront per block, which goes over all rows with their sums known.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void spqt_kv_weigh_kernel(Cache c, Call a) {
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
        if (lanes_max(row.high) < block * kBlock) continue;
        f16x8 q[D / 32];
        const float back = load_queries<D, BF16>(q, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, row.high >= 0, lane);
        const float scale = a.scale * back * kLog2e * scale_k;
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
    float *weights = c.weights + weight_at(c, page, head);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = sum[t][e];
#pragma unroll
            for (int step = 1; step < 16; step *= 2) x += __shfl_xor(x, step);
            const int at = 16 * t + 4 * quarter + e;
            if (column == 0 && block * kBlock + at < length) weights[at] = a.decay == 0.0f ? x : __builtin_fmaf(a.decay, weights[at], x);
        }
}

}  // namespace

extern "C" int spqt_kv_workspace_bytes(int sequences, int rows, int q_heads, int kv_heads, int head_dim, int max_blocks, size_t *out_bytes) {
    if (!out_bytes) return SPQT_EINVAL;
    if (sequences < 1 || sequences > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || kv_heads > 16384 || q_heads < kv_heads || q_heads % kv_heads != 0 ||
        head_dim < 64 || head_dim > SPQT_KV_MAX_DIM || head_dim % 64 != 0 || max_blocks < 1 || max_blocks > 1 << 24)
        return SPQT_ESHAPE;
    *out_bytes = kWorkspaceHead;
    return SPQT_OK;
}

extern "C" int spqt_kv_attention(const spqt_kv_cache *cache, const spqt_kv_rows *q, const spqt_kv_rows *out, float *lse, int rows, const int32_t *counts,
                                 int q_heads, float scale, int window, float decay, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_cache(cache, false);
    if (rc == SPQT_OK) rc = check_rows(q);
    if (rc == SPQT_OK) rc = check_rows(out);
    if (rc != SPQT_OK) return rc;
    size_t need = 0;
    rc = spqt_kv_workspace_bytes(cache->sequences, rows, q_heads, cache->kv_heads, cache->head_dim, cache->max_blocks, &need);
    if (rc != SPQT_OK) return rc;
    if (!workspace || window < 0 || scale != scale || decay != decay || (cache->weights && !lse)) return SPQT_EINVAL;
    if ((uintptr_t)lse % 4 != 0 || (uintptr_t)counts % 4 != 0 || (uintptr_t)workspace % 256 != 0) return SPQT_EALIGN;
    if (workspace_bytes < need) return SPQT_ESIZE;
    const Call a = {view(*q), view(*out), lse, counts, rows, q_heads, q_heads / cache->kv_heads, window, scale, decay};
    if ((int64_t)rows * a.group > 1 << 28) return SPQT_ESHAPE;
    const dim3 grid((rows * a.group + 15) / 16, cache->kv_heads, cache->sequences);
    dispatch(*cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        constexpr bool B = decltype(bf16)::value;
        hipLaunchKernelGGL((spqt_kv_attend_kernel<D, B>), grid, dim3(kThreads), 0, (hipStream_t)stream, view(*cache), a);
        if (cache->weights)
            hipLaunchKernelGGL((spqt_kv_weigh_kernel<D, B>), dim3((cache->max_blocks + kWaves - 1) / kWaves, cache->kv_heads, cache->sequences), dim3(kThreads), 0,
                               (hipStream_t)stream, view(*cache), a);
    });
    return launched();
}
