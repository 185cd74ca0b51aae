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
// gate / (1 + exp(-gate)) * up by the hardware's power of two and reciprocal. The divisor is in sixteenths: the instruction gives 0 in place of
// reciprocals under 2^-126, which those of gates from -87.4 on would be. Where 1 + exp(-gate) leaves fp32, from -88.8 on, the quotient is 0 (with 16
// bits from -90.2 on).
// Halves of fp32's steps that it may be off by: for 16-bit outputs 1.3 |gate| + 11, of the exponential's argument most of them, which are nothing next to
// half a step of the output. For 32-bit ones (WIDE) what the argument lost is a factor of the power: 8, and 4 more where the reciprocal is subnormal.
// 4001 x 28672 x 4096 / 6396 x 8192 x 698 with the gate, 32-bit outputs: 421 / 76 us; with the argument as it is 417 / 73, with expf and a division 441 / 89.
template <bool WIDE>
__device__ __forceinline__ float gated_by(float gate, float up) {
    constexpr float kLog2 = 1.44269502f, kLog2Rest = 1.92596303e-8f, kLn2 = 0.69314718f;
    float sixteenths;
    if (WIDE) {
        const float least = __builtin_amdgcn_fmed3f(gate, -128.0f, 128.0f), power = -least * kLog2;       // (infinities would leave no rest)
        const float rest = __builtin_fmaf(-least, kLog2Rest, __builtin_fmaf(-least, kLog2, -power));
        sixteenths = __builtin_fmaf(__builtin_amdgcn_exp2f(power), __builtin_fmaf(rest, kLn2 / 16, 0.0625f), 0.0625f);
    } else {
        sixteenths = __builtin_amdgcn_exp2f(__builtin_fmaf(gate, -kLog2, -4.0f)) + 0.0625f;
    }
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
