// spqt_i8_gemm: checks, and which kernel a call takes.
#include "i8_gemm.hpp"

using namespace spqt;
using namespace spqt::i8;

extern "C" int spqt_i8_workspace_bytes(int64_t rows, int64_t N, int64_t K, size_t *out_bytes) {
    if (!out_bytes) return SPQT_EINVAL;
    if (N < 1 || N > 1 << 24) return SPQT_ESHAPE;
    const int rc = check_extents(rows, K, SPQT_I8_MAX_K);
    if (rc != SPQT_OK) return rc;
    const size_t sums = most_sums(rows, N, K);
    *out_bytes = sums ? kWorkspaceHead + sums : 0;
    return SPQT_OK;
}

extern "C" int spqt_i8_gemm(const spqt_i8_product *c, void *workspace, size_t workspace_bytes, void *stream) {
    if (!c || (c->gated != 0 && c->gated != 1) || (c->y_type != SPQT_I8_FP32 && !sixteen_bits(c->y_type))) return SPQT_EINVAL;
    size_t need;
    int rc = spqt_i8_workspace_bytes(c->rows, c->N, c->K, &need);
    if (rc != SPQT_OK) return rc;
    if (c->gated && c->N % 2 != 0) return SPQT_ESHAPE;
    const int64_t outputs = c->gated ? c->N / 2 : c->N;
    rc = check_codes(c->codes, c->codes_row, c->rows, c->K, false);
    if (rc == SPQT_OK) rc = check_codes(c->weights, c->weights_row, c->N, c->K, false);
    if (rc == SPQT_OK) rc = check_scales(c->scales);
    if (rc == SPQT_OK) rc = check_scales(c->weight_scales);
    if (rc == SPQT_OK && c->bias) rc = check_scales(c->bias);
    if (rc == SPQT_OK) rc = check_matrix(c->y, c->y_row, c->rows, outputs, c->y_type == SPQT_I8_FP32 ? 4 : 2, true);
    if (rc != SPQT_OK) return rc;
    if (workspace && (uintptr_t)workspace % 256 != 0) return SPQT_EALIGN;
    if (workspace && workspace_bytes < need) return SPQT_ESIZE;
    const Product p = {c->codes, c->weights, c->scales, c->weight_scales, c->bias, c->y, c->codes_row, c->weights_row, c->y_row,
                       (int)c->rows, (int)c->N, (int)c->K, (int)outputs, c->y_type};
    const Plan plan = plan_of(p, c->gated != 0, workspace && need ? need - kWorkspaceHead : 0);
    if (plan.shape >= 0) launch_tiles_of(plan, p, c->gated != 0, workspace, (hipStream_t)stream);
    else launch_few(p, c->gated != 0, (hipStream_t)stream);
    return launched();
}
