// What the attention kernels share: a call, its rows and what each of them sees, and how partial sums of rows join.
#ifndef SPQT_KV_ATTEND_HPP
#define SPQT_KV_ATTEND_HPP

#include "kv_common.hpp"

namespace spqt {
namespace kv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();
// A row's sums of values are put down in units of 2^(its maximum + kRoom): those of 2^30 tokens of bf16's largest number are within fp32's range.
constexpr int kRoom = 32;
// Probabilities go to the matrix instructions as two fp16 numbers, 22 bits in all, the largest of them about 2^15 (kv_units.hpp): fp16's smallest number is 2^-39 of that.

// Query heads of a kv head: places of rows are worked out by the fp32 inverse of it (kv_weigh.hip), exactly up to some 2^21.
constexpr int kMaxGroup = 1 << 20;

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

// What the rows' sums over some tokens and over others make together: (top, total, x) with x in units of 2^(top + kRoom).
struct Meeting {
    float top = kNone, total = 0.0f;
    __device__ __forceinline__ void add(float other_top, float other_total, float &mine, float &others) {
        const float most = __builtin_fmaxf(top, other_top), from = most == kNone ? 0.0f : most;
        mine = __builtin_amdgcn_exp2f(top - from);
        others = __builtin_amdgcn_exp2f(other_top - from);
        total = total * mine + other_total * others;
        top = most;
    }
    __device__ __forceinline__ float inverse() const { return total == 0.0f ? 0.0f : 0x1p32f / total; }
    __device__ __forceinline__ float lse() const { return total == 0.0f ? kNone : (top == kNone ? 0.0f : top) * kLn2 + __builtin_logf(total); }
};

// A negative scale is taken as a positive one for the negative queries, so that the largest score is that of the largest product.
template <int N>
__device__ __forceinline__ float positive_scale(float scale, u32x4 (&w)[N]) {
    const uint32_t flip = as_u32(scale) >> 31 ? 0x80008000u : 0u;
#pragma unroll
    for (int j = 0; j < N; ++j) w[j] ^= flip;
    return __builtin_fabsf(scale);
}

// A lane's part of a row of Q in fp16; `step` is the first distance between the lanes that share the row.  bf16 rows are scaled by a power of two to have
// their largest element in 2^14 .. 2^15, where fp16 holds them (exactly, down to 2^-30 of the largest); the factor that undoes it is returned.
template <bool BF16, int N>
__device__ __forceinline__ float queries_f16(const u32x4 (&w)[N], f16x8 (&q)[N], int step) {
    if (!BF16) {
#pragma unroll
        for (int j = 0; j < N; ++j) q[j] = __builtin_bit_cast(f16x8, w[j]);
        return 1.0f;
    }
    uint32_t largest = 0;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = w[j][e] & 0x7FFFu, y = w[j][e] >> 16 & 0x7FFFu;
            largest = largest > x ? largest : x;
            largest = largest > y ? largest : y;
        }
    for (; step < 64; step *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)largest, step);
        largest = o > largest ? o : largest;
    }
    // exponent field of the largest, kept where 2^(141 - e) and its inverse are numbers; an infinity or a NaN stays what it is
    const int e = clamped((int)(largest >> 7), 20, 254);
    const float up = as_float((uint32_t)(268 - e) << 23), down = as_float((uint32_t)(e - 14) << 23);
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int x = 0; x < 8; ++x) q[j][x] = (_Float16)(as_float(x % 2 ? w[j][x / 2] & 0xFFFF0000u : w[j][x / 2] << 16) * up);
    return down;
}


// 16 rows at a time: S^T = K Q^T, so that a lane of v_mfma_f32_16x16x32_f16 has ONE row of Q and four tokens of each 16.

// f over the 16 rows; the same for all of them.
template <class F>
__device__ __forceinline__ int over_rows(int v, F f) {
    v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x121, 0xf, 0xf, false));                     // row_ror:1, 2, 4, 8
    v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x122, 0xf, 0xf, false));
    v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x124, 0xf, 0xf, false));
    return f(v, __builtin_amdgcn_update_dpp(v, v, 0x128, 0xf, 0xf, false));
}
__device__ __forceinline__ int rows_max(int v) {
    return over_rows(v, [](int x, int y) { return x > y ? x : y; });
}
__device__ __forceinline__ int rows_min(int v) {
    return over_rows(v, [](int x, int y) { return x < y ? x : y; });
}
__device__ __forceinline__ float rows_sum(float v) {
    return as_float((uint32_t)over_rows((int)as_u32(v), [](int x, int y) { return (int)as_u32(as_float((uint32_t)x) + as_float((uint32_t)y)); }));
}
// Over the four lanes of a row.
__device__ __forceinline__ float columns_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
    v = __builtin_fmaxf(as_float(r[0]), as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(as_u32(v), as_u32(v), false, false);
    return __builtin_fmaxf(as_float(r[0]), as_float(r[1]));
}
__device__ __forceinline__ float columns_sum(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
    v = as_float(r[0]) + as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(as_u32(v), as_u32(v), false, false);
    return as_float(r[0]) + as_float(r[1]);
}

// A row of Q as an operand, 32 elements a step: step j of a lane are elements 64 (j / 2) + 16 (lane / 16) + 8 (j % 2) on, as in load_keys; queries_f16 makes it fp16.
template <int D>
__device__ __forceinline__ void load_queries(u32x4 (&w)[D / 32], const uint16_t *row, bool live, int lane) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
        w[j] = live ? *reinterpret_cast<const u32x4 *>(row + 64 * (j / 2) + 16 * (lane / 16) + 8 * (j % 2)) : u32x4{0u, 0u, 0u, 0u};
}

// 16 tokens' keys as an operand.
template <int D>
__device__ __forceinline__ void load_keys(u32x4 (&k)[D / 64], const uint8_t *page, int tile, int lane) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) k[j] = *reinterpret_cast<const u32x4 *>(page + (16 * tile + lane % 16) * D + 64 * j + 16 * (lane / 16));
}

// The products of 16 tokens' codes with the queries.  (The stored bytes as fp16's smallest numbers, 2^-24 (code + 128), would save half of the conversion and
// start the sums at -128 times that of the queries, but a token of small codes in a block of large ones then has the errors of large ones.)
template <int D>
__device__ __forceinline__ f32x4 scores_of(const u32x4 (&k)[D / 64], const f16x8 (&q)[D / 32]) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(u32x2{k[j / 2][2 * (j % 2)], k[j / 2][2 * (j % 2) + 1]}), q[j], s, 0, 0, 0);
    return s;
}

// Partial sums stay in the workspace when a call is done, where a GEMV's exchange takes every word that is not 0 for one of its own.  So each call raises the poison flag that makes GEMVs
// on the workspace give NaN (word 0 of its head): the two kinds of calls have workspaces of their own.
__device__ __forceinline__ void poison_for_gemv(uint32_t *workspace) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) *workspace = 1u;
}

// A few rows (kv_step.hip): what such calls need of the workspace, zeros first, and the call.
constexpr size_t kStepCounters = 1024;                    // bytes of counters at the head of the workspace, all 0 between calls
size_t step_bytes(int dim);                               // and what follows them
bool step_fits(const spqt_kv_cache &cache, const Call &a);
void launch_step(const spqt_kv_cache &cache, const Call &a, void *workspace, void *counters, void *space, hipStream_t stream);

// Many rows (kv_prompt.hip): whether a call is of that kind, what such calls need of the workspace at most, and the call.
constexpr int kFewRows = 64;                              // of a kv head, that are a few in any call
bool is_prompt(int sequences, int rows, int group, int kv_heads, int dim, int max_blocks);
size_t prompt_bytes(int dim);
void launch_prompt(const spqt_kv_cache &cache, const Call &a, void *workspace, void *space, hipStream_t stream);

// What every token weighed in a call whose sums are known (kv_weigh.hip).
void launch_weigh(const spqt_kv_cache &cache, const Call &a, hipStream_t stream);

}  // namespace kv
}  // namespace spqt
#endif
