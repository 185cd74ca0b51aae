// What the kernels of the product in 8-bit integers share: the call, and what becomes of a sum.
#ifndef SPQT_I8_GEMM_HPP
#define SPQT_I8_GEMM_HPP

#include "i8_common.hpp"
#include "i8_plan.hpp"

namespace spqt {
namespace i8 {

// A sum of channel n and a row with this scale. Each step is rounded, here and where the tiles' outputs are made, so that all ways give the same bits.
__device__ __forceinline__ float scaled(const Product &p, int sum, float scale, int n) {
#pragma clang fp contract(off)
    float v = (float)sum * scale * p.weight_scales[n];
    if (p.bias) v += p.bias[n];
    return v;
}
// gate / (1 + exp(-gate)) * up. For 32-bit outputs step by step. For 16 bits by the hardware's power of two and reciprocal, off by 1.3 |gate| + 11 halves of fp32's
// steps at most, which are nothing next to half a step of the output. The divisor is in sixteenths: the instruction gives 0 in place of reciprocals under 2^-126,
// which those of gates from -87.4 on would be. Where 1 + exp(-gate) leaves fp32, from -88.8 on, the quotient is 0 (with 16 bits from -90.2 on).
template <bool WIDE>
__device__ __forceinline__ float gated_by(float gate, float up) {
    if (WIDE) return gate / (1.0f + expf(-gate)) * up;
    const float sixteenths = __builtin_amdgcn_exp2f(__builtin_fmaf(gate, -1.44269504f, -4.0f)) + 0.0625f;
    return gate * (__builtin_amdgcn_rcpf(sixteenths) * 0.0625f) * up;
}

__device__ __forceinline__ void store_one(const Product &p, int64_t row, int n, float v) {
    const int64_t at = row * p.y_row + n;
    if (p.y_type == SPQT_I8_FP32) reinterpret_cast<float *>(p.y)[at] = v;
    else reinterpret_cast<uint16_t *>(p.y)[at] = (uint16_t)(p.y_type == SPQT_I8_BF16 ? narrow2<true>(v, v) : narrow2<false>(v, v));
}

// Zeros in place of what is behind a row's K-th byte, in the 16 bytes from k on.
__device__ __forceinline__ i32x4 masked(i32x4 x, int k, int K) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = K - k - 4 * i;
        x[i] = left >= 4 ? x[i] : left <= 0 ? 0 : x[i] & (int)(0xFFFFFFFFu >> (32 - 8 * left));
    }
    return x;
}

void launch_few(const Product &p, bool gated, hipStream_t stream);
void launch_tiles_of(const Plan &plan, const Product &p, bool gated, void *workspace, hipStream_t stream);

}  // namespace i8
}  // namespace spqt
#endif
