// The product in 8-bit integers, few rows or little of everything: each weight goes from memory to the matrix instruction of one wavefront.
//
// With the weights as its first operand v_mfma_i32_16x16x64_i8 gives a lane four channels of one row. The wavefronts of a workgroup take K in turn,
// 128 bytes each time, and add their sums up in shared memory: whole numbers, whose order does not matter.
//
// What bounds it: reading the weights. 57344 x 8192 with the gate, one row 82 to 86 us = 5.5 to 5.7 TB/s; 28672 x 4096 25.7 us = 4.6; 6144 x 4096 8.5
// us (a launch in a graph is 2 to 3 of that). A lane takes the 16 bytes that follow its neighbour's, so that an instruction reads whole halves of
// lines: with 32 bytes of a lane one after the other the former was 91 us, 28672 x 4096 30.8. Loads that pass the caches by (non-temporal) 93 and
// 27.0; two chunks on their way for four 81.8 and 26.0, and 6144 x 4096 8.9; 16 wavefronts 81.1 and 25.8.
#include "i8_gemm.hpp"

namespace {

using namespace spqt;
using namespace spqt::i8;

constexpr int kChunk = 128;

// W wavefronts, 16 R rows, 16 C channels (gated: half of them the gate's, half of them those of the up projection), D chunks of a wavefront on their
// way together.
template <int W, int R, int C, int D, bool GATED>
__global__ __launch_bounds__(W * 64) void spqt_i8_few_kernel(Product p) {
    constexpr int kMade = GATED ? C / 2 : C;                      // sixteens of outputs
    __shared__ i32x4 sums[W][C * R][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * (16 * kMade), row0 = blockIdx.y * (16 * R);
    const int8_t *a[R], *w[C];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * 16 + line;
        a[r] = p.codes + (row < p.rows ? row : p.rows - 1) * p.codes_row;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        int n = n0 + c % kMade * 16 + line;
        n = (n < p.outputs ? n : p.outputs - 1) + c / kMade * p.outputs;
        w[c] = p.weights + n * p.weights_row;
    }
    i32x4 acc[C][R];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[c][r] = i32x4{0, 0, 0, 0};
    const int whole = p.K / kChunk, chunks = (p.K + kChunk - 1) / kChunk;
    int at = wave;
    auto span = [&](auto deep) {
        constexpr int N = decltype(deep)::value;
        i32x4 x[N][2][R], v[N][2][C];
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = (at + d * W) * kChunk + i * 64 + quarter * 16;
#pragma unroll
                for (int c = 0; c < C; ++c) v[d][i][c] = *reinterpret_cast<const i32x4 *>(w[c] + k);
#pragma unroll
                for (int r = 0; r < R; ++r) x[d][i][r] = *reinterpret_cast<const i32x4 *>(a[r] + k);
            }
        __builtin_amdgcn_sched_barrier(0);                        // all is asked for before any of it is used
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[c][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[d][i][c], x[d][i][r], acc[c][r], 0, 0, 0);
        at += N * W;
    };
    while (at + (D - 1) * W < whole) span(std::integral_constant<int, D>());
    while (at < whole) span(std::integral_constant<int, 1>());
    if (chunks > whole && whole % W == wave) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = whole * kChunk + i * 64 + quarter * 16, from = k < p.K ? k : 0;       // (behind the row's end nothing is read)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const i32x4 x = masked(*reinterpret_cast<const i32x4 *>(a[r] + from), k, p.K);
#pragma unroll
                for (int c = 0; c < C; ++c) acc[c][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(w[c] + from), x, acc[c][r], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) sums[wave][c * R + r][lane] = acc[c][r];
    __syncthreads();
    // a wavefront finishes sixteen outputs of sixteen rows
    static_assert(kMade * R <= W);
    const int row = row0 + wave % R * 16 + line, made = wave / R;
    if (made >= kMade || row >= p.rows) return;
    auto total = [&](int c) {
        i32x4 t = sums[0][c][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) t += sums[i][c][lane];
        return t;
    };
    const i32x4 first = total(wave), second = total(GATED ? wave + kMade * R : wave);
    const float scale = p.scales[row];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + made * 16 + 4 * quarter + e;
        if (n >= p.outputs) break;
        float v = scaled(p, first[e], scale, n);
        if (GATED) {
            const float up = scaled(p, second[e], scale, n + p.outputs);
            v = p.y_type == SPQT_I8_FP32 ? gated_by<true>(v, up) : gated_by<false>(v, up);
        }
        store_one(p, row, n, v);
    }
}

template <int W, int R, int C, int D, bool GATED>
void launch(const Product &p, hipStream_t stream) {
    const int made = 16 * (GATED ? C / 2 : C), most = 65535 * 16;                               // rows of a grid
    for (int64_t first = 0; first < p.rows; first += most) {
        Product part = p;
        part.rows = (int)(p.rows - first < most ? p.rows - first : most);
        part.codes += first * p.codes_row;
        part.scales += first;
        part.y = (uint8_t *)p.y + first * p.y_row * (p.y_type == SPQT_I8_FP32 ? 4 : 2);
        hipLaunchKernelGGL((spqt_i8_few_kernel<W, R, C, D, GATED>), dim3((p.outputs + made - 1) / made, (part.rows + 16 * R - 1) / (16 * R)), dim3(W * 64), 0, stream, part);
    }
}

}  // namespace

namespace spqt {
namespace i8 {

// Sixteen channels a workgroup, thirty-two where sixteen rows' codes are so many that reading them for every sixteen channels counts, and there are
// workgroups enough all the same. Rows x channels x K, us of 16 / 32 channels:
//   at the rule's bound of 112 K codes    4 x 8192 x 28672 44.9 / 44.0      8 x 8192 x 14336 28.1 / 26.2      12 x 57344 x 8192 with the gate (96 K) 98.2 / 94.3
//   over it    16 x 8192 x 28672 61.2 / 47.1      16 x 57344 x 8192 with the gate 105 / 100      16 x 8192 x 8192 20.8 / 18.9
//   under it   4 x 8192 x 8192 17.0 / 17.9      8 x 57344 x 8192 with the gate 91.9 / 95.4      1 x 28672 x 4096 24.7 / 28.7      1 x 57344 x 8192 with the gate 84.0 / 92.7
// Under it and without the gate the other way round from 8 to 12 rows on, by up to 12 %: 8 x 14336 x 4096 18.4 / 17.2, 16 x 28672 x 4096 33.9 / 30.3. Few workgroups:
// 16 x 4096 x 14336 19.7 / 24.1.
void launch_few(const Product &p, bool gated, hipStream_t stream) {
    if (p.rows > 32) return gated ? launch<8, 4, 2, 1, true>(p, stream) : launch<8, 4, 1, 1, false>(p, stream);
    if (p.rows > 16) return gated ? launch<8, 2, 2, 2, true>(p, stream) : launch<8, 2, 1, 2, false>(p, stream);
    const bool wide = (int64_t)p.rows * p.K >= 112 << 10 && p.outputs >= 256 * 32;
    if (gated) wide ? launch<8, 1, 4, 2, true>(p, stream) : launch<8, 1, 2, 4, true>(p, stream);
    else wide ? launch<8, 1, 2, 2, false>(p, stream) : launch<8, 1, 1, 4, false>(p, stream);
}

}  // namespace i8
}  // namespace spqt
