// Rows of numbers to 8-bit codes and back, and the norms before and after a block (spqt_i8.h has the definitions).
#include "i8_common.hpp"

#include <utility>

namespace {

using namespace spqt;
using namespace spqt::i8;

// T threads hold a row of up to 8 T V numbers, thread t the eights t, t + T, ...; rows of one wavefront share a workgroup of four.
template <int T>
struct Shape {
    static constexpr int kThreads = T == 64 ? 256 : T, kRows = kThreads / T, kWaves = T / 64;
};

template <int T>
__device__ __forceinline__ int place(int v) {
    return ((int)(threadIdx.x % T) + v * T) * 8;
}

// Rows of whole 512s (WHOLE) end between two wavefronts' eights: whether a wavefront has its v-th ones is one question for all its lanes, and nothing
// needs to be moved or masked. With that question asked lane by lane 4001 rows of 8192 took a norm 56 us in place of 53, 20000 of 512 22.4 in place
// of 19.1, and codes of 4001 rows of 14336 34.5 in place of 32.5.
template <int T, bool WHOLE>
__device__ __forceinline__ bool has(int v, int K) {
    if (!WHOLE) return place<T>(v) < K;
    return (__builtin_amdgcn_readfirstlane((int)(threadIdx.x % T) / 64) * 64 + v * T) * 8 < K;
}

// Eight 16-bit numbers from element k on, as they lie. At a row's end the row's last eight, which settle() moves to their places, with 0 from element
// K on; rows of less than eight are put together from single ones.
template <int T, bool WHOLE>
__device__ __forceinline__ u32x4 fetch(const uint16_t *row, int v, int K) {
    const int k = place<T>(v);
    if (WHOLE) return *reinterpret_cast<const u32x4_at2 *>(row + (has<T, WHOLE>(v, K) ? k : k % 512));
    if (T == 64 && K < 8) {
        u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (k == 0 && e < K) w[e / 2] |= (uint32_t)row[e] << (16 * (e % 2));
        return w;
    }
    return *reinterpret_cast<const u32x4_at2 *>(row + (k + 8 <= K ? k : K - 8));
}
template <int T, bool WHOLE>
__device__ __forceinline__ u32x4 settle(u32x4 w, int v, int K) {
    if (WHOLE) return has<T, WHOLE>(v, K) ? w : u32x4{0u, 0u, 0u, 0u};
    const int k = place<T>(v);
    if (k + 8 <= K || (T == 64 && K < 8)) return w;
    const int by = k + 8 - K < 8 ? k + 8 - K : 8;                 // elements that are not this thread's, in front
    const uint32_t odd = by & 1;
    uint32_t x[5] = {w.x, w.y, w.z, w.w, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = odd ? __builtin_amdgcn_alignbyte(x[i + 1], x[i], 2) : x[i];
    const int whole = by >> 1;
    if (whole & 1) w = u32x4{w.y, w.z, w.w, 0u};
    if (whole & 2) w = u32x4{w.z, w.w, 0u, 0u};
    if (whole & 4) w = u32x4{0u, 0u, 0u, 0u};
    return w;
}
template <bool BF16>
__device__ __forceinline__ void widen8(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = widen<BF16>(w[e / 2] >> (16 * (e % 2)) & 0xFFFFu);
}
template <bool BF16, bool WHOLE>
__device__ __forceinline__ void put(uint16_t *row, int k, int K, const float (&x)[8]) {
    const u32x4 w = {narrow2<BF16>(x[0], x[1]), narrow2<BF16>(x[2], x[3]), narrow2<BF16>(x[4], x[5]), narrow2<BF16>(x[6], x[7])};
    if (WHOLE || k + 8 <= K) {
        *reinterpret_cast<u32x4_at2 *>(row + k) = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (k + e < K) row[k + e] = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
}

// A value of every thread of a row together, 0 leaving any other as it is: over the lanes of a wavefront first, then the wavefronts' through shared
// memory, `slot` being another one than the last time.
template <int T, class F>
__device__ __forceinline__ uint32_t over_row(uint32_t v, F f, uint32_t *shared, int slot) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));      // row_shr:1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));      // row_bcast:15
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));      // row_bcast:31
    v = (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
    if (T == 64) return v;
    constexpr int kWaves = T / 64;
    if (threadIdx.x % 64 == 0) shared[slot * kWaves + threadIdx.x / 64] = v;
    __syncthreads();
    uint32_t all = shared[slot * kWaves];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = f(all, shared[slot * kWaves + w]);
    return all;
}
template <int T>
__device__ __forceinline__ float sum_over_row(float v, uint32_t *shared, int slot) {
    return as_float(over_row<T>(as_u32(v), [](uint32_t a, uint32_t b) { return as_u32(as_float(a) + as_float(b)); }, shared, slot));
}
template <int T>
__device__ __forceinline__ uint32_t most_over_row(uint32_t v, uint32_t *shared, int slot) {
    return over_row<T>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }, shared, slot);
}

// 1 / sqrt(mean x^2 + eps), within 3.5 halves of fp32's steps behind the sum: 1 / K and its product, the sum with eps, these by the root's half, and
// two of the hardware's reciprocal root. Where the mean is over 2^252 the result is a subnormal number, 4 more of them. Squares of numbers from 2^64
// on, and sums of 2^16 of them from 2^56 on, leave fp32, as mean + eps may: such a row is summed in units of 2^80, in which its largest number is
// from 2^-24 to 2^48, or eps is 2^-33 and more.
template <int T, int V>
__device__ __forceinline__ float inverse_rms(const float (&x)[V][8], float per, float eps, uint32_t *shared, int slot) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[v][e], x[v][e], sum);
    sum = sum_over_row<T>(sum, shared, slot);
    const float mean = sum * per + eps;
    if (mean < __builtin_inff() || mean != mean) return __builtin_amdgcn_rsqf(mean);
    sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = x[v][e] * 0x1p-80f;
            sum = __builtin_fmaf(y, y, sum);
        }
    sum = sum_over_row<T>(sum, shared, slot + 1);
    return 0x1p-80f * __builtin_amdgcn_rsqf(sum * per + eps * 0x1p-80f * 0x1p-80f);
}

// Codes of a row, from the largest magnitude of this thread's numbers: magnitudes order as their bits do, infinities and NaN above all numbers.
template <int T, int V, bool WHOLE>
__device__ __forceinline__ void quantize_row(const float (&x)[V][8], int K, int8_t *codes, float *scale, uint32_t *shared, int slot) {
#pragma clang fp contract(off)
    uint32_t most = 0u;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t m = as_u32(x[v][e]) & 0x7FFFFFFFu;
            most = m > most ? m : most;
        }
    most = most_over_row<T>(most, shared, slot);
    const bool number = most < 0x7F800000u;
    const float top = __builtin_fmaxf(as_float(most), 0x1p-100f), inverse = 127.0f / top;
    if (threadIdx.x % T == 0) *scale = number ? top / 127.0f : __builtin_nanf("");
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!has<T, WHOLE>(v, K)) continue;
        const int k = place<T>(v);
        u32x2 w;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // the product rounded, then 1.5 2^23 added, which rounds it to the nearest integer: the code is in the lowest byte
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = as_u32(x[v][4 * i + j] * inverse + 12582912.0f);
            w[i] = __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
            if (!number) w[i] = 0u;
        }
        if (WHOLE || k + 8 <= K) {
            *reinterpret_cast<u32x2 *>(codes + k) = w;
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (k + e < K) codes[k + e] = (int8_t)(w[e / 4] >> (8 * (e % 4)));
        }
    }
}

struct Quantize {
    const uint16_t *x;
    int8_t *codes;
    float *scales;
    int64_t x_row, codes_row;
    int rows, K;
};

// A row is in the registers of its threads: read once, its largest magnitude found, its codes written.
// What bounds it: 2 bytes in and 1 out a number. Call after call over tensors of 860 MB, which no cache keeps: 4001 rows of 14336 32.5 us = 5.3 TB/s, of
// 8192 20.5 = 4.8 (a copy: 5.1); 300 of 65536 17.7 = 3.3; 40 of 28672 3.7 us; one of 4096 2.1. In turn with calls that read the codes back, which writes
// 115 MB in between, 4001 rows of 14336 take 36 to 38.
template <int T, int V, bool BF16, bool WHOLE>
__global__ __launch_bounds__(Shape<T>::kThreads) void spqt_i8_quantize_kernel(Quantize a) {
    typedef Shape<T> S;
    __shared__ uint32_t shared[2 * S::kWaves];
    int slot = 0;
    for (int64_t row = (int64_t)blockIdx.x * S::kRows + (S::kRows > 1 ? threadIdx.x / T : 0); row < a.rows; row += (int64_t)gridDim.x * S::kRows) {
        float x[V][8];
        u32x4 w[V];
#pragma unroll
        for (int v = 0; v < V; ++v) w[v] = fetch<T, WHOLE>(a.x + row * a.x_row, v, a.K);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = 0; v < V; ++v) widen8<BF16>(settle<T, WHOLE>(w[v], v, a.K), x[v]);
        quantize_row<T, V, WHOLE>(x, a.K, a.codes + row * a.codes_row, a.scales + row, shared, slot);
        slot ^= 1;
    }
}

struct Norm {
    const uint16_t *h, *block, *block_gain, *gate, *gain;
    uint16_t *h_out, *out;
    int8_t *codes;
    float *scales;
    int64_t h_row, block_row, gate_row, h_out_row, out_row, codes_row;
    int rows, K;
    float residual, eps, offset, per;              // per: 1 / K
};

// One pass: what a block has made, the stream and the vectors are read once, and the sum stays in registers, in 32 bits, from the join over both
// norms to the codes. TOGETHER: everything is asked for before any of it is used. That takes half as many registers again, with which a CU holds
// fewer wavefronts: of 512 and 1024 threads, two workgroups and one in place of four and two. Together / not: one row of 8192 4.2 / 4.7 us, 40 rows
// 4.5 / 5.1, 256 rows 6.3 / 6.8, 512 rows 9.2 / 8.9, 4001 rows 53.0 / 48.1; 300 rows of 14336 13.1 / 10.8, 1000 rows 33.7 / 26.6; of 256 threads,
// 4001 rows of 4096 26.5 / 27.4. What bounds it: 4 bytes in and 3 out a number, and three sums over a row that follow each other: 4001 rows of 8192
// with both norms and a gate 48 us = 4.8 TB/s; with sums over lanes by way of shared memory 82. One row of 4096 3.7 us: loads, three sums, stores.
// Rows of more than 32768 have more numbers than registers (17 to 163 of them in scratch memory): 300 rows of 65536 59 us = 2.3 TB/s, two 14.6 us;
// 300 of 32768 27 us = 2.5 TB/s.
template <int T, int V, bool BF16, bool WHOLE, bool TOGETHER>
__global__ __launch_bounds__(Shape<T>::kThreads) void spqt_i8_norm_kernel(Norm a) {
    typedef Shape<T> S;
    __shared__ uint32_t shared[5 * S::kWaves];
    for (int64_t row = (int64_t)blockIdx.x * S::kRows + (S::kRows > 1 ? threadIdx.x / T : 0); row < a.rows; row += (int64_t)gridDim.x * S::kRows) {
        u32x4 h[V], block[V], block_gain[V], gate[V], gain[V];
        const uint16_t *const h_at = a.h + row * a.h_row, *const gate_at = a.gate + row * a.gate_row;
        auto fetch_row = [&](u32x4 (&w)[V], const uint16_t *from) {
#pragma unroll
            for (int v = 0; v < V; ++v) w[v] = fetch<T, WHOLE>(from, v, a.K);
        };
        if (a.block) fetch_row(block, a.block + row * a.block_row);
        if (TOGETHER) {
            fetch_row(h, h_at);
            if (a.block_gain) fetch_row(block_gain, a.block_gain);
            if (a.gate) fetch_row(gate, gate_at);
            fetch_row(gain, a.gain);
            __builtin_amdgcn_sched_barrier(0);
        }
        auto numbers = [&](const u32x4 (&w)[V], const uint16_t *from, int v, float (&x)[8]) {
            widen8<BF16>(settle<T, WHOLE>(TOGETHER ? w[v] : fetch<T, WHOLE>(from, v, a.K), v, a.K), x);
        };
        auto gains = [&](const u32x4 (&w)[V], const uint16_t *from, int v, float (&x)[8]) {
            numbers(w, from, v, x);
            if (a.offset != 0.0f)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += a.offset;
        };
        float s[V][8], other[8];
        if (a.block) {
#pragma unroll
            for (int v = 0; v < V; ++v) widen8<BF16>(settle<T, WHOLE>(block[v], v, a.K), s[v]);
            if (a.block_gain) {
                const float by = inverse_rms<T, V>(s, a.per, a.eps, shared, 0);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    gains(block_gain, a.block_gain, v, other);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[v][e] = s[v][e] * by * other[e];
                }
            }
            if (a.gate)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    numbers(gate, gate_at, v, other);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[v][e] *= other[e];
                }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                numbers(h, h_at, v, other);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[v][e] = __builtin_fmaf(a.residual, other[e], s[v][e]);
                if (has<T, WHOLE>(v, a.K)) put<BF16, WHOLE>(a.h_out + row * a.h_out_row, place<T>(v), a.K, s[v]);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) numbers(h, h_at, v, s[v]);
        }
        const float by = inverse_rms<T, V>(s, a.per, a.eps, shared, 2);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            gains(gain, a.gain, v, other);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[v][e] = s[v][e] * by * other[e];
            if (a.out && has<T, WHOLE>(v, a.K)) put<BF16, WHOLE>(a.out + row * a.out_row, place<T>(v), a.K, s[v]);
        }
        if (a.codes) quantize_row<T, V, WHOLE>(s, a.K, a.codes + row * a.codes_row, a.scales + row, shared, 4);
        if (T > 64) __syncthreads();               // the slots are free again
    }
}

// What codes stand for: eight a thread. 1 byte in and 2 out: 4001 rows of 14336 33.8 us = 5.1 TB/s from memory (860 MB in turn), 27 to 28 where the codes
// were just written and are partly in the cache behind memory.
struct Read {
    const int8_t *codes;
    const float *scales;
    uint16_t *out;
    int64_t codes_row, out_row;
    int rows, K, per_row;                          // workgroups a row
};
template <bool BF16>
__global__ __launch_bounds__(256) void spqt_i8_read_kernel(Read a) {
    const float largest = BF16 ? as_float(0x7F7F0000u) : 65504.0f;
    for (int64_t unit = blockIdx.x; unit < (int64_t)a.rows * a.per_row; unit += gridDim.x) {
        const int64_t row = unit / a.per_row;
        const int k = ((int)(unit - row * a.per_row) * 256 + (int)threadIdx.x) * 8;
        if (k >= a.K) continue;
        const float scale = a.scales[row];
        const u32x2 w = *reinterpret_cast<const u32x2 *>(a.codes + row * a.codes_row + k);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = (float)((int)(w[e / 4] << (24 - 8 * (e % 4))) >> 24) * scale;
            x[e] = v != v ? v : __builtin_fmaxf(-largest, __builtin_fminf(v, largest));
        }
        put<BF16, false>(a.out + row * a.out_row, k, a.K, x);
    }
}

// f(threads, eights a thread, BF16, whole 512s) for rows of K numbers: a norm's threads hold two eights up to where a workgroup ends, since they have
// five tensors to ask for. With rows' ends asked for lane by lane, codes of 4001 rows of 14336 with 512 x 4 / 1024 x 2 / 256 x 8 34.4 / 40.3 / 35.9
// us, of 8192 with 256 x 4 / 512 x 2 / 1024 x 1 20.5 / 21.2 / 24.2; norms of 4001 rows of 4096 with 256 x 2 / 512 x 1 27.8 / 34.5.
template <bool NORM, class F>
void dispatch(int64_t K, int type, F f) {
    auto typed = [&](auto t, auto v) {
        auto whole = [&](auto bf16) {
            if (K % 512 == 0) f(t, v, bf16, std::true_type());
            else f(t, v, bf16, std::false_type());
        };
        if (type == SPQT_I8_BF16) whole(std::true_type());
        else whole(std::false_type());
    };
    if (K <= 512) typed(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (K <= 2048) typed(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    else if (K <= 4096) typed(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    else if (K <= 8192) typed(std::integral_constant<int, NORM ? 512 : 256>(), std::integral_constant<int, NORM ? 2 : 4>());
    else if (K <= 16384) typed(std::integral_constant<int, NORM ? 1024 : 512>(), std::integral_constant<int, NORM ? 2 : 4>());
    else if (K <= 32768) typed(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
    else typed(std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
}
template <class S>
dim3 grid_of(int64_t rows) {
    const int64_t n = (rows + S::kRows - 1) / S::kRows;
    return dim3((unsigned)(n < 1 << 20 ? n : 1 << 20));
}

}  // namespace

extern "C" int spqt_i8_quantize(const void *x, int64_t x_row, int64_t rows, int64_t K, int type, int8_t *codes, int64_t codes_row, float *scales, void *stream) {
    if (!sixteen_bits(type)) return SPQT_EINVAL;
    int rc = check_extents(rows, K, SPQT_I8_MAX_NORM);
    if (rc == SPQT_OK) rc = check_matrix(x, x_row, rows, K, 2, false);
    if (rc == SPQT_OK) rc = check_codes(codes, codes_row, rows, K, true);
    if (rc == SPQT_OK) rc = check_scales(scales);
    if (rc != SPQT_OK) return rc;
    const Quantize a = {(const uint16_t *)x, codes, scales, x_row, codes_row, (int)rows, (int)K};
    dispatch<false>(K, type, [&](auto t, auto v, auto bf16, auto whole) {
        typedef Shape<decltype(t)::value> S;
        hipLaunchKernelGGL((spqt_i8_quantize_kernel<decltype(t)::value, decltype(v)::value, decltype(bf16)::value, decltype(whole)::value>), grid_of<S>(rows), dim3(S::kThreads), 0,
                           (hipStream_t)stream, a);
    });
    return launched();
}

extern "C" int spqt_i8_read(const int8_t *codes, int64_t codes_row, const float *scales, int64_t rows, int64_t K, int type, void *out, int64_t out_row, void *stream) {
    if (!sixteen_bits(type)) return SPQT_EINVAL;
    int rc = check_extents(rows, K, SPQT_I8_MAX_K);
    if (rc == SPQT_OK) rc = check_codes(codes, codes_row, rows, K, false);
    if (rc == SPQT_OK) rc = check_scales(scales);
    if (rc == SPQT_OK) rc = check_matrix(out, out_row, rows, K, 2, true);
    if (rc != SPQT_OK) return rc;
    const int per_row = (int)((K + 2047) / 2048);
    const int64_t units = rows * per_row;
    const Read a = {codes, scales, (uint16_t *)out, codes_row, out_row, (int)rows, (int)K, per_row};
    const dim3 grid((unsigned)(units < 1 << 22 ? units : 1 << 22));
    if (type == SPQT_I8_BF16) hipLaunchKernelGGL(spqt_i8_read_kernel<true>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(spqt_i8_read_kernel<false>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return launched();
}

extern "C" int spqt_i8_norm(const spqt_i8_norm_call *c, void *stream) {
    if (!c || !sixteen_bits(c->type) || (!c->codes && !c->out && !c->h_out)) return SPQT_EINVAL;
    if (!c->block != !c->h_out || (!c->block && (c->block_gain || c->gate)) || !c->codes != !c->scales) return SPQT_EINVAL;
    if (!(c->eps >= 1e-30f) || !__builtin_isfinite(c->eps) || !__builtin_isfinite(c->residual) || !__builtin_isfinite(c->offset)) return SPQT_EINVAL;
    if (c->h_out && c->h_out == c->out) return SPQT_EINVAL;
    const int64_t rows = c->rows, K = c->K;
    // in place means element for element: other rows' workgroups may not read what one of them writes
    for (const auto &w : {std::make_pair(c->h_out, c->h_out_row), std::make_pair(c->out, c->out_row)}) {
        const auto clash = [&](const void *read, int64_t row) { return w.first && w.first == read && rows > 1 && w.second != row; };
        if (clash(c->h, c->h_row) || clash(c->block, c->block_row) || clash(c->gate, c->gate_row) || clash(c->gain, 0) || clash(c->block_gain, 0)) return SPQT_EINVAL;
    }
    int rc = check_extents(rows, K, SPQT_I8_MAX_NORM);
    if (rc == SPQT_OK) rc = check_matrix(c->h, c->h_row, rows, K, 2, false);
    if (rc == SPQT_OK) rc = check_matrix(c->gain, 0, 1, K, 2, false);
    if (rc == SPQT_OK && c->block) rc = check_matrix(c->block, c->block_row, rows, K, 2, false);
    if (rc == SPQT_OK && c->block_gain) rc = check_matrix(c->block_gain, 0, 1, K, 2, false);
    if (rc == SPQT_OK && c->gate) rc = check_matrix(c->gate, c->gate_row, rows, K, 2, false);
    if (rc == SPQT_OK && c->h_out) rc = check_matrix(c->h_out, c->h_out_row, rows, K, 2, true);
    if (rc == SPQT_OK && c->out) rc = check_matrix(c->out, c->out_row, rows, K, 2, true);
    if (rc == SPQT_OK && c->codes) rc = check_codes(c->codes, c->codes_row, rows, K, true);
    if (rc == SPQT_OK && c->codes) rc = check_scales(c->scales);
    if (rc != SPQT_OK) return rc;
    const Norm a = {(const uint16_t *)c->h, (const uint16_t *)c->block, (const uint16_t *)c->block_gain, (const uint16_t *)c->gate, (const uint16_t *)c->gain,
                    (uint16_t *)c->h_out, (uint16_t *)c->out, c->codes, c->scales, c->h_row, c->block_row, c->gate_row, c->h_out_row, c->out_row, c->codes_row,
                    (int)rows, (int)K, c->residual, c->eps, c->offset, 1.0f / (float)K};
    dispatch<true>(K, c->type, [&](auto t, auto v, auto bf16, auto whole) {
        constexpr int T = decltype(t)::value, V = decltype(v)::value;
        auto launch = [&](auto together) {
            hipLaunchKernelGGL((spqt_i8_norm_kernel<T, V, decltype(bf16)::value, decltype(whole)::value, decltype(together)::value>), grid_of<Shape<T>>(rows), dim3(Shape<T>::kThreads), 0,
                               (hipStream_t)stream, a);
        };
        // together while a CU has a row at most, where nothing else runs beside a load's way, and always where that leaves wavefronts enough
        if constexpr (V > 2) launch(std::false_type());
        else if constexpr (T < 512) launch(std::true_type());
        else rows <= 256 ? launch(std::true_type()) : launch(std::false_type());
    });
    return launched();
}
