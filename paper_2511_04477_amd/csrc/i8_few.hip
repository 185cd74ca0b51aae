// The product in 8-bit integers, sixteen rows at a time: each weight goes from memory to the matrix instruction of one wavefront.
//
// With the weights as its first operand v_mfma_i32_16x16x64_i8 gives a lane four channels of one row. K goes in chunks of 128 bytes, of which a lane has 32:
// which of them are which is the same for both operands, so any order will do. The wavefronts of a workgroup take the chunks in turn and add their sums up in shared memory.
#include "i8_gemm.hpp"

namespace {

using namespace spqt;
using namespace spqt::i8;

constexpr int kWaves = 8, kChunk = 128;

template <bool GATED>
__global__ __launch_bounds__(kWaves * 64) void spqt_i8_few_kernel(Product p) {
    constexpr int C = GATED ? 2 : 1;
    __shared__ i32x4 sums[kWaves][C][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * 16, row0 = blockIdx.y * 16;
    const int row = row0 + line < p.rows ? row0 + line : p.rows - 1;
    const int8_t *a = p.codes + row * p.codes_row, *w[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int n = n0 + line < p.outputs ? n0 + line : p.outputs - 1;
        w[c] = p.weights + (int64_t)(n + c * p.outputs) * p.weights_row;
    }
    i32x4 acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = i32x4{0, 0, 0, 0};
    const int whole = p.K / kChunk, chunks = (p.K + kChunk - 1) / kChunk;
    for (int at = wave; at < whole; at += kWaves) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = at * kChunk + quarter * 32 + i * 16;
            const i32x4 x = *reinterpret_cast<const i32x4 *>(a + k);
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(w[c] + k), x, acc[c], 0, 0, 0);
        }
    }
    if (chunks > whole && whole % kWaves == wave) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = whole * kChunk + quarter * 32 + i * 16, from = k < p.K ? k : 0;       // (behind the row's end nothing is read)
            const i32x4 x = masked(*reinterpret_cast<const i32x4 *>(a + from), k, p.K);
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(w[c] + from), x, acc[c], 0, 0, 0);
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) sums[wave][c][lane] = acc[c];
    __syncthreads();
    if (wave > 0 || row0 + line >= p.rows) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
        for (int i = 1; i < kWaves; ++i) acc[c] += sums[i][c][lane];
    const float scale = p.scales[row];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + 4 * quarter + e;
        if (n >= p.outputs) break;
        float v = scaled(p, acc[0][e], scale, n);
        if (GATED) v = gated_by(v, scaled(p, acc[C - 1][e], scale, n + p.outputs));
        store_one(p, row, n, v);
    }
}

}  // namespace

namespace spqt {
namespace i8 {

void launch_few(const Product &p, bool gated, hipStream_t stream) {
    const dim3 grid((p.outputs + 15) / 16, (p.rows + 15) / 16);
    if (gated) hipLaunchKernelGGL(spqt_i8_few_kernel<true>, grid, dim3(kWaves * 64), 0, stream, p);
    else hipLaunchKernelGGL(spqt_i8_few_kernel<false>, grid, dim3(kWaves * 64), 0, stream, p);
}

}  // namespace i8
}  // namespace spqt
