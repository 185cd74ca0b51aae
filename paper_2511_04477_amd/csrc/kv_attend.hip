// spqt_kv_attention: attention of some rows over the cache, and what every cached token weighed in it.  A few rows go to kv_step.hip, many to kv_prompt.hip.
#include "kv_attend.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

constexpr int kThreads = 256, kWaves = kThreads / 64;

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

}  // namespace

extern "C" int spqt_kv_workspace_bytes(int sequences, int rows, int q_heads, int kv_heads, int head_dim, int max_blocks, size_t *out_bytes) {
    if (!out_bytes) return SPQT_EINVAL;
    if (sequences < 1 || sequences > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || kv_heads > 16384 || q_heads < kv_heads || q_heads % kv_heads != 0 ||
        head_dim < 64 || head_dim > SPQT_KV_MAX_DIM || head_dim % 64 != 0 || max_blocks < 1 || max_blocks > 1 << 24)
        return SPQT_ESHAPE;
    const int group = q_heads / kv_heads;
    if ((int64_t)rows * group > 1 << 28) return SPQT_ESHAPE;
    // one kind of call's partial sums or the other's
    size_t bytes = step_bytes(head_dim);
    if (is_prompt(rows, group) && prompt_bytes(head_dim) > bytes) bytes = prompt_bytes(head_dim);
    *out_bytes = kWorkspaceHead + kStepCounters + bytes;
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
    const bool prompt = is_prompt(rows, a.group);
    if (!prompt && !step_fits(*cache, a)) return SPQT_ESHAPE;
    char *counters = (char *)workspace + kWorkspaceHead, *space = counters + kStepCounters;
    if (prompt) launch_prompt(*cache, a, space, (hipStream_t)stream);
    else launch_step(*cache, a, counters, space, (hipStream_t)stream);
    if (!cache->weights) return launched();
    dispatch(*cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        constexpr bool B = decltype(bf16)::value;
        hipLaunchKernelGGL((spqt_kv_weigh_kernel<D, B>), dim3((cache->max_blocks + kWaves - 1) / kWaves, cache->kv_heads, cache->sequences), dim3(kThreads), 0,
                           (hipStream_t)stream, view(*cache), a);
    });
    return launched();
}
