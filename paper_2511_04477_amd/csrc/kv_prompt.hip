// Attention of many rows over the cache: a workgroup takes 256 (128) of a kv head's rows and goes through the blocks of tokens that they see; the codes of a
// block are made fp16 once, in shared memory, for all of them.
//
// With S^T = K Q^T a lane of v_mfma_f32_32x32x16_f16 has one row of Q and half of each 32 tokens, and what it has of P^T is an operand of
// O^T = V^T P^T if a line of V^T holds the tokens in that order: per 16 tokens the fours 0 and 2 for the lower lanes, 1 and 3 for the upper ones.
//
// Probabilities go to the matrix instructions as two fp16 numbers, 22 bits in all, as they do where rows are few: what a row gets does not depend on which kernel a call takes.  One number
// would save a third of the products' instructions (4001 rows of 32 / 8 heads of 128 166 us for 208, 1024 rows over 32768 tokens 1042 for 1397), and every output would be off by up to 2^-11
// of sum p |v|: against 64 bits 2.5e-4 of an fp16 output instead of the 2.1e-4 of its own rounding.
//
// What bounds it: matrix and vector instructions of a SIMD side by side; a block takes a SIMD's two wavefronts 96 matrix instructions of 32 cycles and about 810 others, most of them for
// the softmax and its two numbers (the matrix units are busy for 0.56 of the time, the vector units for 0.72).  1024 rows of 64 / 8 heads of 128 over 32768 tokens 1397 to 1520 us, by the
// card, = 0.72 to 0.77 PFLOP/s (1.08 to 1.16 of what the instructions multiply; an 8192^3 product: 1.2); 4001 rows of 32 / 8 heads from an empty cache 208 to 220 us, since 504 workgroups of
// uneven length on 256 CUs leave some idle at the end.
#include "kv_attend.hpp"
#include "kv_units.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Eight wavefronts of 32 rows, two on every SIMD; four where sums and queries of longer heads leave no registers for two.
template <int D>
struct Shape {
    static constexpr int kThreads = D > 128 ? 256 : 512, kWaves = kThreads / 64, kRows = kWaves * 32;
    static constexpr int kKeyStride = D + 8, kValueStride = kBlock + 8;      // fp16 numbers; 16 lines are in 16 different sets of banks
};

// Heads of 128 have no registers left for what the compiler keeps from before the loop, places in shared and global memory: it would lie in scratch memory, which every turn waits for
// (1024 rows of 64 / 8 heads over 32768 tokens 1707 us for 1397; heads of 64 145 for 156, of 256 261 for 267 the other way round).
template <int D>
__device__ __forceinline__ int worked_out_anew(int v) {
    if (D == 128) asm("" : "+v"(v));
    return v;
}

// A thread's part of a block's keys or values, on its way from codes to numbers.
template <int D>
struct StagedKeys {
    static constexpr int kThreads = Shape<D>::kThreads, kParts = (D * 4 + kThreads - 1) / kThreads;
    u32x4 part[kParts];                  // 16 elements of a token

    template <class F>
    __device__ __forceinline__ void each(F f) {
        const int thread = worked_out_anew<D>(threadIdx.x);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int at = thread + i * kThreads;
            if (D * 4 % kThreads == 0 || at < D * 4) f(part[i], at);
        }
    }
    __device__ __forceinline__ void fetch(const uint8_t *page) {
        each([&](u32x4 &x, int at) { x = *reinterpret_cast<const u32x4 *>(page + at * 16); });
    }
    __device__ __forceinline__ void put_down(_Float16 *k) {
        each([&](u32x4 &x, int at) {
            _Float16 *to = k + at / (D / 16) * Shape<D>::kKeyStride + at % (D / 16) * 16;
            *reinterpret_cast<f16x8 *>(to) = codes_f16(u32x2{x.x, x.y});
            *reinterpret_cast<f16x8 *>(to + 8) = codes_f16(u32x2{x.z, x.w});
        });
    }
};
template <int D>
struct StagedValues {
    static constexpr int kThreads = Shape<D>::kThreads, kParts = (D * 4 + kThreads - 1) / kThreads;
    u32x2 part[kParts][2];               // of one element: fours 0 and 2, or 1 and 3, of two of the block's 16s

    template <class F>
    __device__ __forceinline__ void each(F f) {
        const int thread = worked_out_anew<D>(threadIdx.x);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int at = thread + i * kThreads;
            if (D * 4 % kThreads == 0 || at < D * 4) f(part[i], at / 4, at / 2 % 2, at % 2);
        }
    }
    __device__ __forceinline__ void fetch(const uint8_t *page) {
        each([&](u32x2 (&x)[2], int d, int half, int pair) {
#pragma unroll
            for (int y = 0; y < 2; ++y) x[y] = *reinterpret_cast<const u32x2 *>(page + kBlock * D + d * kBlock + (half + 2 * y) * 16 + pair * 8);
        });
    }
    __device__ __forceinline__ void put_down(_Float16 *v) {
        each([&](u32x2 (&x)[2], int d, int half, int pair) {
            _Float16 *to = v + d * Shape<D>::kValueStride + pair * 32 + half * 8;
            *reinterpret_cast<f16x8 *>(to) = codes_f16(u32x2{x[0].x, x[1].x});
            *reinterpret_cast<f16x8 *>(to + 16) = codes_f16(u32x2{x[0].y, x[1].y});
        });
    }
};

__device__ __forceinline__ float halves_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(as_u32(v), as_u32(v), false, false);
    return __builtin_fmaxf(as_float(r[0]), as_float(r[1]));
}

// Where the tokens are divided into parts: what each of them makes of a row, in units of 2^(its maximum + kRoom).
struct Parts {
    int n;
    uint32_t *head;      // of the workspace
    float *sums;         // [sequence][kv head][256 (128) rows][part][row][D]
    float *stats;        // the same of [2]: a row's maximum and sum
};

// Waits for the workgroup's shared memory, not for what is on its way from global memory.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The wavefronts of a SIMD take turns: while the first four's products run, O += V P of one block and S = K Q of the next, the other four work out the
// probabilities of theirs, and the other way round.  In the latter turn a wavefront also makes its part of the next block's codes numbers:
//
//   turn        2b                              2b + 1
//   first four  O += V P(b-1), S = K(b) Q       P(b), K(b+1), V(b)
//   others      P(b-1), K(b+1), V(b)            O += V P(b-1), S = K(b) Q
template <int D, bool BF16>
__global__ __launch_bounds__(Shape<D>::kThreads) void spqt_kv_prompt_kernel(Cache c, Call a, int tiles, Parts parts) {
    typedef Shape<D> S;
    __shared__ __attribute__((aligned(16))) _Float16 keys[2][kBlock * S::kKeyStride];
    __shared__ __attribute__((aligned(16))) _Float16 values[2][D * S::kValueStride];
    // heads first: workgroups of one head run on one XCD if there are eight; the rows that see most first
    const int s = blockIdx.z, head = blockIdx.x % c.kv_heads, tile = tiles - 1 - (int)(blockIdx.x / c.kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = lane & 31, half = lane >> 5;
    const int length = length_of(c, s), count = count_of(a.counts, s, a.rows), rows = a.rows * a.group;
    poison_for_gemv(parts.head);

    // the blocks that any row of the workgroup sees
    const int r0 = tile * S::kRows;
    const Row first = row_of(a, r0, head, length, count);
    const int last_live = r0 + S::kRows < count * a.group ? r0 + S::kRows - 1 : count * a.group - 1;
    const Row last = row_of(a, last_live < 0 ? 0 : last_live, head, length, count);
    const bool any = last_live >= r0 && last.high >= 0;
    const int whole_begin = any ? block_of(first.high >= 0 ? first.low : 0) : 0, whole = any ? block_of(last.high) + 1 - whole_begin : 0;
    // this workgroup's part of them
    const int from_block = (int)((int64_t)whole * blockIdx.y / parts.n), begin = whole_begin + from_block;
    const int n = (int)((int64_t)whole * (blockIdx.y + 1) / parts.n) - from_block;

    const int r = r0 + wave * 32 + column;
    Row row = row_of(a, r, head, length, count);
    if (r >= rows) row.high = -1;
    f16x8 q[D / 16];
    float scale, total = 0.0f, shrink = 1.0f;
    BlockUnits units;
    units.start();
    {
        const bool live = row.high >= 0;
        const uint16_t *from = a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head;
        u32x4 w[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) w[j] = live ? *reinterpret_cast<const u32x4 *>(from + 16 * j + 8 * half) : u32x4{0u, 0u, 0u, 0u};
        scale = positive_scale(a.scale, w) * kLog2e;
        scale *= queries_f16<BF16>(w, q, 32);
    }
    int full_low = row.low, full_high = row.high;             // every row of the wavefront sees these tokens
#pragma unroll
    for (int step = 1; step < 32; step *= 2) {
        const int l = __shfl_xor(full_low, step), h = __shfl_xor(full_high, step);
        full_low = l > full_low ? l : full_low;
        full_high = h < full_high ? h : full_high;
    }
    full_low = __builtin_amdgcn_readfirstlane(full_low);
    full_high = __builtin_amdgcn_readfirstlane(full_high);
    f32x16 acc[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};

    // Pages and scales of 64 blocks from `base` on, one per lane: looked up rarely, so that no turn waits for a chain of loads.
    const int32_t *table = c.table + (size_t)s * c.max_blocks + begin;
    uint32_t places = 0;                                      // of the page and head among all pages' heads: their codes are within the memory there is
    float scales_k = 0.0f, scales_v = 0.0f, inverses_v = 0.0f;             // (1 / the part from 1/2 to 1 of scales_v)
    int base = 0;
    auto look_up = [&](int b) {
        base = b;
        const int at = b + lane < n ? b + lane : n - 1;
        uint32_t page = (uint32_t)table[at];
        const bool there = page < c.pages;
        if (!there) page = 0;
        places = page * (uint32_t)c.kv_heads + (uint32_t)head;
        scales_k = there ? c.scales[scale_at(c, page, head, 0)] : __builtin_nanf("");
        scales_v = there ? c.scales[scale_at(c, page, head, 1)] : __builtin_nanf("");
        inverses_v = 1.0f / __builtin_amdgcn_frexp_mantf(scales_v);
    };
    auto codes_of = [&](int b) { return c.codes + (size_t)lane_of(places, b - base) * (2 * kBlock * D); };
    auto scalar = [&](float v, int b) { return as_float(lane_of(as_u32(v), b - base)); };

    f32x16 p[2];
    f16x8 lifted[4], rest[4];                                // probabilities and what their first number leaves
    // O += V P of the last block and S = K Q of this one: kProducts matrix instructions in a row, whose other operands are read kAhead ahead.
    // A wavefront alone on its SIMD goes through the values 32 elements at a time and brings the next 32's sums to their new units beside those products: 4001 rows of 16 / 4 heads of
    // 256 299 -> 227 us, of 192 184 -> 182.  Where two take turns the one that multiplies has no time for it: heads of 128 174 for 171, of 64 136 for 133.
    constexpr int kAhead = 6, kValueProducts = D / 8, kProducts = kValueProducts + D / 8;
    constexpr bool kBeside = S::kWaves == 4;
    auto tile_of = [](int i) { return kBeside ? i / 4 : i % (D / 32); };      // 32 elements and 16 tokens of the i-th product with values
    auto sixteen_of = [](int i) { return kBeside ? i % 4 : i / (D / 32); };
    auto products = [&](const _Float16 *v, const _Float16 *k, auto skip, auto stop) {
        constexpr int from = decltype(skip)::value ? kValueProducts : 0, to = decltype(stop)::value ? kValueProducts : kProducts;
        f16x8 x[kAhead];
        const int here = worked_out_anew<D>(lane);
        const int line = here & 31, part = here >> 5 << 3;
        auto read = [&](int i) {
            if (i < kValueProducts) return *reinterpret_cast<const f16x8 *>(v + (tile_of(i) * 32 + line) * S::kValueStride + sixteen_of(i) * 16 + part);
            i -= kValueProducts;
            return *reinterpret_cast<const f16x8 *>(k + (i % 2 * 32 + line) * S::kKeyStride + i / 2 * 16 + part);
        };
#pragma unroll
        for (int i = from; i < from + kAhead; ++i) x[i % kAhead] = read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = from; i < to; ++i) {
            if (i < kValueProducts) {
                acc[tile_of(i)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % kAhead], lifted[sixteen_of(i)], acc[tile_of(i)], 0, 0, 0);
                acc[tile_of(i)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % kAhead], rest[sixteen_of(i)], acc[tile_of(i)], 0, 0, 0);
                if (kBeside && i + 4 < kValueProducts)
#pragma unroll
                    for (int e = 4 * (i % 4); e < 4 * (i % 4) + 4; ++e) acc[i / 4 + 1][e] *= shrink;
            } else {
                const int t = (i - kValueProducts) % 2, j = (i - kValueProducts) / 2;
                p[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % kAhead], q[j], j == 0 ? f32x16{} : p[t], 0, 0, 0);
            }
            if (i + kAhead < to) x[i % kAhead] = read(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto probabilities = [&](int block, float scale_k, float scale_v, float inverse_v, auto masked) {
        const float by = scale * scale_k;
        if (decltype(masked)::value) {
            uint32_t first = (uint32_t)(block * kBlock + 4 * half - row.low);
            const uint32_t seen = row.high < row.low ? 0u : (uint32_t)(row.high - row.low) + 1u;
            asm("" : "+v"(first));                            // else the 32 tokens' places are kept in registers from before the loop
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (first + (uint32_t)(32 * t + 8 * (e / 4) + e % 4) >= seen) p[t][e] = kNone;
        }
        float most = p[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = __builtin_fmaxf(most, p[t][e]);
        most = halves_max(most);
        const BlockUnits::Step step = units.see(!decltype(masked)::value || !(most == kNone), most * by, __builtin_amdgcn_frexp_mantf(scale_v), inverse_v, (float)__builtin_amdgcn_frexp_expf(scale_v));
        total *= step.total;
        shrink = step.sums;
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                f32x2 x;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(p[t][e + i], by, -step.less));
                    x[i] = decltype(masked)::value && p[t][e + i] == kNone ? 0.0f : y;
                    sum += x[i];
                }
                const f16x2 h = __builtin_convertvector(x, f16x2);
                const f16x2 l = __builtin_convertvector(f32x2{x[0] - (float)h[0], x[1] - (float)h[1]}, f16x2);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    lifted[2 * t + e / 8][e % 8 + i] = h[i];
                    rest[2 * t + e / 8][e % 8 + i] = l[i];
                }
            }
        total += sum * step.back;
#pragma unroll
        for (int i = 0; i < (kBeside ? 1 : D / 32); ++i) acc[i] *= shrink;
    };

    if (n > 0) {
        const int later = wave >= 4 ? 1 : 0;
        StagedKeys<D> next_keys;
        StagedValues<D> next_values;
        look_up(0);
        next_keys.fetch(codes_of(0));
        next_keys.put_down(keys[0]);
        next_keys.fetch(codes_of(1));
        next_values.fetch(codes_of(0));
        auto stage = [&](int b) {                             // K(b + 1), V(b)
            next_keys.put_down(keys[(b + 1) & 1]);
            next_values.put_down(values[b & 1]);
            next_keys.fetch(codes_of(b + 2));
            next_values.fetch(codes_of(b + 1));
        };
        if (later) stage(0);
        meet();
        if (later) meet();
        for (int b = 0; b < n; ++b) {
            __builtin_amdgcn_s_setprio(1);
            if (b > 0) products(values[(b - 1) & 1], keys[b & 1], std::false_type(), std::false_type());
            else products(values[0], keys[0], std::true_type(), std::false_type());
            __builtin_amdgcn_s_setprio(0);
            meet();
            if (b + 3 - base >= 64) look_up(b);
            const float scale_k = scalar(scales_k, b), scale_v = scalar(scales_v, b), inverse_v = scalar(inverses_v, b);
            const int block = begin + b;
            if (block * kBlock >= full_low && block * kBlock + kBlock - 1 <= full_high) probabilities(block, scale_k, scale_v, inverse_v, std::false_type());
            else probabilities(block, scale_k, scale_v, inverse_v, std::true_type());
            stage(b + later);
            if (!later || b + 1 < n) meet();
        }
        products(values[(n - 1) & 1], keys[0], std::false_type(), std::true_type());
    }

    Meeting sum;
    sum.top = units.top;
    const auto both = __builtin_amdgcn_permlane32_swap(as_u32(total), as_u32(total), false, false);
    sum.total = as_float(both[0]) + as_float(both[1]);
    const int drop = units.drop() - kRoom;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = __builtin_ldexpf(acc[i][e] * units.part, drop);
    if (parts.n > 1) {
        const size_t slot = ((((size_t)s * c.kv_heads + head) * tiles + tile) * parts.n + blockIdx.y) * S::kRows + wave * 32 + column;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(parts.sums + slot * D + 32 * i + 2 * e + 4 * half) = f32x4{acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]};
        if (half == 0) *reinterpret_cast<f32x2 *>(parts.stats + slot * 2) = f32x2{sum.top, sum.total};
        return;
    }
    if (r >= rows) return;
    uint16_t *out = a.out.data + s * a.out.sequence + row.i * a.out.row + row.head * a.out.head + 4 * half;
    const float by = sum.inverse();
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            *reinterpret_cast<u32x2 *>(out + 32 * i + 2 * e) =
                u32x2{narrow2_within<BF16>(acc[i][e] * by, acc[i][e + 1] * by), narrow2_within<BF16>(acc[i][e + 2] * by, acc[i][e + 3] * by)};
        }
    if (a.lse && half == 0) a.lse[((size_t)s * a.rows + row.i) * a.q_heads + row.head] = sum.lse();
}

// The parts' sums of a row to its output, eight rows a workgroup.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void spqt_kv_parts_kernel(Call a, int kv_heads, int tiles, Parts parts) {
    constexpr int kEach = D / 32;
    const int s = blockIdx.z, head = blockIdx.y, r = blockIdx.x * 8 + threadIdx.x / 32, d = threadIdx.x % 32 * kEach;
    if (r >= a.rows * a.group) return;
    const size_t slot = (((size_t)s * kv_heads + head) * tiles + r / Shape<D>::kRows) * parts.n * Shape<D>::kRows + r % Shape<D>::kRows;
    Meeting m;
    float x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = 0.0f;
#pragma unroll 4
    for (int part = 0; part < parts.n; ++part) {
        const size_t at = slot + (size_t)part * Shape<D>::kRows;
        const f32x2 stat = *reinterpret_cast<const f32x2 *>(parts.stats + at * 2);
        float mine, others;
        m.add(stat.x, stat.y, mine, others);
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = x[i] * mine + parts.sums[at * D + d + i] * others;
    }
    const int i = r / a.group, q_head = head * a.group + r % a.group;
    uint16_t *out = a.out.data + s * a.out.sequence + i * a.out.row + q_head * a.out.head + d;
    const float by = m.inverse();
#pragma unroll
    for (int e = 0; e < kEach; e += 2) *reinterpret_cast<uint32_t *>(out + e) = narrow2_within<BF16>(x[e] * by, x[e + 1] * by);
    if (a.lse && threadIdx.x % 32 == 0) a.lse[((size_t)s * a.rows + i) * a.q_heads + q_head] = m.lse();
}

constexpr int kParted = 256;                              // workgroups of a launch whose tokens are divided, at most
// Parts that the tokens are divided into, where the rows alone would not fill the chip: as many as leave one workgroup per CU, of at least eight
// blocks each for a sequence that fills its table.
int parts_of(int64_t units, int max_blocks) {
    int64_t n = kParted / units;
    if (n > max_blocks / 8) n = max_blocks / 8;
    return n < 1 ? 1 : (n > 64 ? 64 : (int)n);
}
int rows_of(int dim) { return dim > 128 ? Shape<256>::kRows : Shape<128>::kRows; }

}  // namespace

namespace spqt {
namespace kv {

// Up to 64 rows of a kv head are a few.  Up to 512 are, in sixteens, where that makes few blocks to go through (with the room of the tables), at most as many as 24000 of 128
// elements; as 65536 where the rows fill no more than 5/8 of what the workgroups here would take.  As a few / here, heads of 128: 80, 256 and 512 rows of each of 8 over 4000 tokens
// (2500, 8000, 16000 blocks) 16.5 / 41.5, 23.5 / 38.1, 31.0 / 41.6 us; 256 over 16000 and 32000 (32000, 64000) 53 / 45, 95 / 65; not full: 128 rows over 32000, 64000 and 131000 (32000,
// 64000, 131000) 53 / 63, 100 / 109, 235 / 204, 80 over 131000 (82000) 166 / 223, 160 over 64000 (80000) 125 / 112.  Heads of 192, full: 16000 44 / 47, 32000 69 / 63, not: 40000 89 / 118; of 256, full: 16000 51 / 54, 32000 98 / 83,
// not: 20000 86 / 82; of 64, full: 128000 115 / 86, not: 80000 73 / 100.
// Sixteens of a few blocks have to have a workgroup each (their start and end count): 640 sixteens of 3 blocks 18.6 / 16.1, 4096 of 5 40.6 / 28.4, 2560 of 5 33.4 / 26.8 (but 1024 of 3 15.2 / 20.0).
bool is_prompt(int sequences, int rows, int group, int kv_heads, int dim, int max_blocks) {
    const int64_t all = (int64_t)rows * group, sixteens = (all + 15) / 16, tiles = (all + rows_of(dim) - 1) / rows_of(dim), units = (int64_t)sequences * kv_heads * sixteens;
    const int limit = 8 * 16 * sixteens <= 5 * tiles * rows_of(dim) ? 65536 : 24000;
    return all > 512 || (all > kFewRows && ((units > 256 && max_blocks < 8) || units * max_blocks > limit * 128 / dim));
}

size_t prompt_bytes(int dim) { return (size_t)kParted * rows_of(dim) * (dim + 2) * 4; }

void launch_prompt(const spqt_kv_cache &cache, const Call &a, void *workspace, void *space, hipStream_t stream) {
    dispatch(cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        constexpr bool B = decltype(bf16)::value;
        const int tiles = (a.rows * a.group + Shape<D>::kRows - 1) / Shape<D>::kRows;
        const int64_t units = (int64_t)tiles * cache.kv_heads * cache.sequences;
        Parts parts;
        parts.n = parts_of(units, cache.max_blocks);
        parts.head = (uint32_t *)workspace;
        parts.sums = (float *)space;
        parts.stats = parts.sums + (size_t)units * parts.n * Shape<D>::kRows * D;
        hipLaunchKernelGGL((spqt_kv_prompt_kernel<D, B>), dim3((unsigned)tiles * cache.kv_heads, parts.n, cache.sequences), dim3(Shape<D>::kThreads), 0, stream,
                           view(cache), a, tiles, parts);
        if (parts.n > 1)
            hipLaunchKernelGGL((spqt_kv_parts_kernel<D, B>), dim3((a.rows * a.group + 7) / 8, cache.kv_heads, cache.sequences), dim3(256), 0, stream, a, cache.kv_heads,
                               tiles, parts);
    });
}

}  // namespace kv
}  // namespace spqt
