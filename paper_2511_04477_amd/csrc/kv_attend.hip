// spqt_kv_attention: attention of some rows over the cache, and what every cached token weighed in it.  A few rows go to kv_step.hip, many to kv_prompt.hip;
// what the tokens weighed is kv_weigh.hip's.
#include "kv_attend.hpp"

using namespace spqt;
using namespace spqt::kv;

extern "C" int spqt_kv_workspace_bytes(int sequences, int rows, int q_heads, int kv_heads, int head_dim, int max_blocks, size_t *out_bytes) {
    if (!out_bytes) return SPQT_EINVAL;
    if (sequences < 1 || sequences > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || kv_heads > 16384 || q_heads < kv_heads || q_heads % kv_heads != 0 ||
        head_dim < 64 || head_dim > SPQT_KV_MAX_DIM || head_dim % 64 != 0 || max_blocks < 1 || max_blocks > 1 << 24)
        return SPQT_ESHAPE;
    const int group = q_heads / kv_heads;
    if ((int64_t)rows * group > 1 << 28 || group > kMaxGroup) return SPQT_ESHAPE;
    // either kind of call's partial sums, whatever the room of the tables, so that a workspace for more sequences, rows or blocks serves less of them
    size_t bytes = step_bytes(head_dim);
    if ((int64_t)rows * group > kFewRows && prompt_bytes(head_dim) > bytes) bytes = prompt_bytes(head_dim);
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
    if (!workspace || window < 0 || scale != scale || decay != decay || (cache->weights && (!lse || q->data == out->data))) return SPQT_EINVAL;
    if ((uintptr_t)lse % 4 != 0 || (uintptr_t)counts % 4 != 0 || (uintptr_t)workspace % 256 != 0) return SPQT_EALIGN;
    if (workspace_bytes < need) return SPQT_ESIZE;
    const Call a = {view(*q), view(*out), lse, counts, rows, q_heads, q_heads / cache->kv_heads, window, scale, decay};
    const bool prompt = is_prompt(cache->sequences, rows, a.group, cache->kv_heads, cache->head_dim, cache->max_blocks);
    if (!prompt && !step_fits(*cache, a)) return SPQT_ESHAPE;
    char *counters = (char *)workspace + kWorkspaceHead, *space = counters + kStepCounters;
    if (prompt) launch_prompt(*cache, a, workspace, space, (hipStream_t)stream);
    else launch_step(*cache, a, workspace, counters, space, (hipStream_t)stream);
    if (cache->weights) launch_weigh(*cache, a, (hipStream_t)stream);
    return launched();
}
