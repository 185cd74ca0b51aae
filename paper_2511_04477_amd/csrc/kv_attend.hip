// spqt_kv_attention: attention of some rows over the cache, softmax statistics of one pass (running maximum and sum), and what
// every cached token weighed in it.
//
// The rows that share a kv head - row i of the call and query head g of the head's group - are numbered r = i * group + g and taken 16 at a
// time.  With S^T = K Q^T a lane of v_mfma_f32_16x16x32_f16 has ONE row of Q and four tokens of each 16, and what it has of P^T is what it
// needs as an operand of O^T = V^T P^T, given the order in which a page holds the values (place_of): probabilities never leave their lane.
// Codes are exact in fp16, so the products are those of the 16-bit queries with the codes; the scale of a block goes into its scores and
// into its probabilities.
#include "kv_attend.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kLeast = 8;                            // blocks that a workgroup takes at least, if there are as many
__device__ __forceinline__ int lanes_max(int v) {            // over the 16 rows
#pragma unroll
    for (int step = 1; step < 16; step *= 2) {
        const int o = __shfl_xor(v, step);
        v = o > v ? o : v;
    }
    return v;
}
__device__ __forceinline__ float columns_max(float v) {      // over the four lanes of a row
    v = __builtin_fmaxf(v, __shfl_xor(v, 16));
    return __builtin_fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float columns_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// A row of Q as an operand, 32 elements a step: step j of a lane are elements 64 (j / 2) + 16 (lane / 16) + 8 (j % 2) on, as in load_keys. Returns queries_f16's factor.
template <int D, bool BF16>
__device__ __forceinline__ float load_queries(f16x8 (&q)[D / 32], const uint16_t *row, bool live, int lane) {
    u32x4 w[D / 32];
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
        w[j] = live ? *reinterpret_cast<const u32x4 *>(row + 64 * (j / 2) + 16 * (lane / 16) + 8 * (j % 2)) : u32x4{0u, 0u, 0u, 0u};
    return queries_f16<BF16>(w, q, 16);
}

// 16 tokens' keys as an operand.
template <int D>
__device__ __forceinline__ void load_keys(u32x4 (&k)[D / 64], const uint8_t *page, int tile, int lane) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) k[j] = *reinterpret_cast<const u32x4 *>(page + (16 * tile + lane % 16) * D + 64 * j + 16 * (lane / 16));
}

template <int D>
__device__ __forceinline__ f32x4 scores_of(const u32x4 (&k)[D / 64], const f16x8 (&q)[D / 32]) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const u32x2 half = {k[j / 2][2 * (j % 2)], k[j / 2][2 * (j % 2) + 1]};
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(half), q[j], s, 0, 0, 0);
    }
    return s;
}

// Where the sums of rows meet: two places for each workgroup, and a counter of what has come for the one unit that begins in it and goes on in others.
struct Space {
    uint32_t *arrived;   // [kShares], all 0 between calls
    float *stats;        // [2 * kShares][16][2]: the rows' maxima and sums
    float *sums;         // [2 * kShares][16][D]
};
constexpr int kShares = 256;                              // workgroups of a launch: one per CU
// Two wavefronts per SIMD, or one where heads of more than 128 elements take its registers: 16 KB of codes in flight each, or 24 or 32.
constexpr int step_threads(int dim) { return dim > 128 ? 256 : 512; }

// A sequence's blocks from the first one that a row sees to its last one; one block, which nobody sees, if there are none.
struct Span {
    int length, count, first, blocks;
};
__device__ __forceinline__ Span span_of(const Cache &c, const Call &a, int s) {
    Span v;
    v.length = length_of(c, s);
    v.count = count_of(a.counts, s, a.rows);
    const int at = v.length > v.count ? v.length - v.count : 0;           // the first row's position
    v.first = a.window > 0 && at >= a.window ? (at - a.window + 1) / kBlock : 0;
    v.blocks = v.length > 0 && v.count > 0 ? (v.length - 1) / kBlock - v.first + 1 : 1;
    if (v.length == 0 || v.count == 0) v.first = 0;
    return v;
}

// Attention of up to 16 rows (of one kv head and sequence) over some of its blocks, by one wavefront: the running statistics and sums.
template <int D, bool BF16>
struct Wave {
    f16x8 q[D / 32];
    Row row;
    float scale, top, total, unit;       // the row's running maximum, this lane's part of its sum, the scale that acc is in
    f32x4 acc[D / 16];
    u32x4 k[4][D / 64], v[D / 16];

    __device__ __forceinline__ void start(const Call &a, const Span &span, int s, int head, int tile, int lane) {
        const int r = tile * 16 + (lane & 15);
        row = row_of(a, r, head, span.length, span.count);
        if (r >= a.rows * a.group) row.high = -1;
        const float back = load_queries<D, BF16>(q, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, row.high >= 0, lane);
        scale = a.scale * back * kLog2e;
        top = kNone;
        total = 0.0f;
        unit = 0x1p-120f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) acc[i] = {0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ __forceinline__ void fetch_keys(const uint8_t *page, int lane) {
#pragma unroll
        for (int t = 0; t < 4; ++t) load_keys<D>(k[t], page, t, lane);
    }
    __device__ __forceinline__ void fetch_values(const uint8_t *page, int lane) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const u32x4 *>(page + (16 * i + (lane & 15)) * kBlock + 16 * (lane >> 4));
    }
    // One block, whose codes have been fetched.  `refill_keys` and `refill_values` request the next one's, each as soon as the registers are free.
    template <class K, class V>
    __device__ __forceinline__ void block(int number, float scale_k, float scale_v, int lane, K refill_keys, V refill_values) {
        f32x4 p[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) p[t] = scores_of<D>(k[t], q);
        refill_keys();
        float most = top;
        const float by = scale * scale_k;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int token = number * kBlock + 16 * t + 4 * (lane >> 4) + e;
                p[t][e] = token >= row.low && token <= row.high ? p[t][e] * by : kNone;
                most = __builtin_fmaxf(most, p[t][e]);
            }
        most = columns_max(most);
        const float from = most == kNone ? 0.0f : most;      // nothing seen yet: 2^(-inf - 0)
        float shrink = __builtin_amdgcn_exp2f(top - from);
        total *= shrink;
        top = most;
        if (scale_v > unit) {
            shrink *= unit / scale_v;
            unit = scale_v;
        }
        const float ratio = scale_v / unit * kLift;
        f16x8 lifted[2], rest[2];                            // a probability in units of `unit`
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool seen = !(p[t][e] == kNone);       // a NaN is one
                const float x = __builtin_amdgcn_exp2f(p[t][e] - from);
                total += x;
                const float y = seen ? x * ratio : 0.0f;
                const _Float16 h = (_Float16)y;
                lifted[t / 2][4 * (t % 2) + e] = h;
                rest[t / 2][4 * (t % 2) + e] = (_Float16)(y - (float)h);
            }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            acc[i] *= shrink;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const f16x8 codes = codes_f16(u32x2{v[i][2 * u], v[i][2 * u + 1]});
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, lifted[u], acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, rest[u], acc[i], 0, 0, 0);
            }
        }
        refill_values();
    }
    // Blocks first .. first + n - 1 of the sequence.  Pages and scales of 64 of them are looked up at once, one per lane.
    __device__ __forceinline__ void blocks(const Cache &c, const Span &span, int s, int head, int first, int n, int lane) {
        const int32_t *table = c.table + (size_t)s * c.max_blocks;
        for (int done = 0; done < n; done += 64) {
            const int b0 = first + done, here = n - done < 64 ? n - done : 64;
            uint32_t page = 0;
            float scales[2] = {__builtin_nanf(""), __builtin_nanf("")};
            if (lane < here && (b0 + lane) * kBlock < span.length) {
                page = (uint32_t)table[b0 + lane];
                if (page < c.pages) {
                    scales[0] = c.scales[scale_at(c, page, head, 0)];
                    scales[1] = c.scales[scale_at(c, page, head, 1)];
                } else {
                    page = 0;
                }
            }
            auto codes_of = [&](int i) { return c.codes + codes_at(c, (uint32_t)__builtin_amdgcn_readlane((int)page, i), head, 0); };
            auto scale_of = [&](int i, int which) { return as_float((uint32_t)__builtin_amdgcn_readlane((int)as_u32(scales[which]), i)); };
            const uint8_t *now = codes_of(0);
            fetch_keys(now, lane);
            fetch_values(now + kBlock * D, lane);
            for (int i = 0; i + 1 < here; ++i) {
                const uint8_t *next = codes_of(i + 1);
                block(b0 + i, scale_of(i, 0), scale_of(i, 1), lane, [&]() { fetch_keys(next, lane); }, [&]() { fetch_values(next + kBlock * D, lane); });
            }
            block(b0 + here - 1, scale_of(here - 1, 0), scale_of(here - 1, 1), lane, []() {}, []() {});
        }
    }
};

// A few rows over the whole cache: up to 16 rows of a kv head and sequence, a unit, share one pass over its blocks.  All units' blocks, in order, are dealt out
// evenly: to the workgroups, and a workgroup's to its wavefronts.  A unit that lies within one wavefront's share is written by it; the parts
// of one that lies within one workgroup's meet in shared memory; those of a longer one in the workspace, where the workgroup that comes last joins
// them, in order.
template <int D, bool BF16>
__global__ __launch_bounds__(step_threads(D)) void spqt_kv_step_kernel(Cache c, Call a, Space space, int sequences, int tiles) {
    constexpr int kStepWaves = step_threads(D) / 64;
    __shared__ float sums[kStepWaves][16][D + 4];
    __shared__ float stats[kStepWaves][2][16];
    __shared__ uint32_t order[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = lane & 15, quarter = lane >> 4;
    const uint32_t units_each = (uint32_t)(c.kv_heads * tiles);          // of a sequence

    // blocks in all
    uint32_t all = 0;
    for (int s0 = 0; s0 < sequences; s0 += 64) {
        uint32_t n = s0 + lane < sequences ? (uint32_t)span_of(c, a, s0 + lane).blocks : 0u;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) n += (uint32_t)__shfl_xor((int)n, step);
        all += n;
    }
    all *= units_each;
    all = (uint32_t)__builtin_amdgcn_readfirstlane((int)all);
    uint32_t shares = (all + kLeast - 1) / kLeast;
    shares = shares < (uint32_t)kShares ? shares : (uint32_t)kShares;
    if (blockIdx.x >= shares) return;
    const uint32_t each = all / shares, more = all % shares;             // the first `more` shares have one block more
    auto begin_of = [&](uint32_t g) { return g * each + (g < more ? g : more); };
    auto share_of = [&](uint32_t block) { return block < more * (each + 1) ? block / (each + 1) : more + (block - more * (each + 1)) / each; };
    const uint32_t group_begin = begin_of(blockIdx.x), group_end = begin_of(blockIdx.x + 1), group_blocks = group_end - group_begin;
    const uint32_t begin = group_begin + group_blocks * (uint32_t)wave / kStepWaves, end = group_begin + group_blocks * (uint32_t)(wave + 1) / kStepWaves;

    // the unit that `block` lies in
    struct Place {
        Span span;
        int s;
        uint32_t unit, start;            // number among the sequence's units; its first block
    };
    auto place_of_block = [&](uint32_t block) {
        uint32_t before = 0, found = 0, in_front = 0;
        for (int s0 = 0; s0 < sequences; s0 += 64) {
            const uint32_t mine = s0 + lane < sequences ? (uint32_t)span_of(c, a, s0 + lane).blocks * units_each : 0u;
            uint32_t upto = mine;
#pragma unroll
            for (int step = 1; step < 64; step *= 2) {
                const uint32_t other = (uint32_t)__shfl_up((int)upto, step);
                upto += lane >= step ? other : 0u;
            }
            const uint64_t past = __ballot(before + upto > block);
            if (past) {
                const int l = __builtin_ctzll(past);
                found = (uint32_t)(s0 + l);
                in_front = before + (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), l);
                break;
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        Place p;
        p.s = (int)found;
        p.span = span_of(c, a, p.s);
        p.unit = (block - in_front) / (uint32_t)p.span.blocks;
        p.start = in_front + p.unit * (uint32_t)p.span.blocks;
        return p;
    };
    auto next_unit = [&](Place &p) {
        p.start += (uint32_t)p.span.blocks;
        if (++p.unit == units_each) {
            p.unit = 0;
            ++p.s;
            if (p.s < sequences) p.span = span_of(c, a, p.s);
        }
    };

    Wave<D, BF16> w;
    // the rows' sums so far, in units of 2^top, to this wavefront's place in shared memory
    auto put_down = [&]() {
        const float total = columns_sum(w.total), drop = w.unit * (1.0f / kLift);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&sums[wave][column][16 * i + 4 * quarter]) = w.acc[i] * drop;
        if (quarter == 0) {
            stats[wave][0][column] = w.top;
            stats[wave][1][column] = total;
        }
    };
    // a lane's row of a unit, from its (whole) sums in registers
    auto write_row = [&](const Place &p, const Meeting &m, const f32x4 (&x)[D / 16], float by) {
        const int r = (int)(p.unit % (uint32_t)tiles) * 16 + column;
        if (r >= a.rows * a.group) return;
        const int i = r / a.group, head = (int)(p.unit / (uint32_t)tiles) * a.group + r % a.group;
        uint16_t *out = a.out.data + p.s * a.out.sequence + i * a.out.row + head * a.out.head + 4 * quarter;
        by *= m.inverse();
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            uint16_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = narrow<BF16>(x[d][e] * by);
            *reinterpret_cast<u32x2 *>(out + 16 * d) = u32x2{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16};
        }
        if (a.lse && quarter == 0) a.lse[((size_t)p.s * a.rows + i) * a.q_heads + head] = m.lse();
    };
    typedef unsigned long long Word;                                      // two numbers, stored and loaded past the XCDs' caches
    auto put_word = [](float *to, float x, float y) {
        __hip_atomic_store(reinterpret_cast<Word *>(to), as_u32(x) | (Word)as_u32(y) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    auto get_word = [](const float *from) { return __hip_atomic_load(reinterpret_cast<const Word *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };

    // a thread's part of a row where all threads work on one unit
    constexpr int kRowThreads = step_threads(D) / 16, kPart = D / kRowThreads;
    const int my_row = threadIdx.x / kRowThreads, my_d = threadIdx.x % kRowThreads * kPart;
    auto write_part = [&](const Place &p, const Meeting &m, const float (&x)[kPart]) {
        const int r = (int)(p.unit % (uint32_t)tiles) * 16 + my_row;
        if (r >= a.rows * a.group) return;
        const int i = r / a.group, head = (int)(p.unit / (uint32_t)tiles) * a.group + r % a.group;
        uint16_t *out = a.out.data + p.s * a.out.sequence + i * a.out.row + head * a.out.head + my_d;
        const float by = m.inverse();
#pragma unroll
        for (int d = 0; d < kPart; d += 2) *reinterpret_cast<uint32_t *>(out + d) = narrow<BF16>(x[d] * by) | (uint32_t)narrow<BF16>(x[d + 1] * by) << 16;
        if (a.lse && threadIdx.x % kRowThreads == 0) a.lse[((size_t)p.s * a.rows + i) * a.q_heads + head] = m.lse();
    };

    const Place group_first = place_of_block(group_begin);
    const bool one_unit = group_end <= group_first.start + (uint32_t)group_first.span.blocks;      // all of the workgroup's blocks
    const bool begins_before = group_first.start < group_begin;
    Place p = group_first;
    if (begin >= group_first.start + (uint32_t)group_first.span.blocks && begin < end) p = place_of_block(begin);
    bool open = false;                                                    // sums of a unit that goes on in the next wavefront are in registers
    for (uint32_t at = begin; at < end;) {
        const uint32_t stop = p.start + (uint32_t)p.span.blocks, upto = stop < end ? stop : end;
        const int head = (int)(p.unit / (uint32_t)tiles);
        w.start(a, p.span, p.s, head, (int)(p.unit % (uint32_t)tiles), lane);
        w.blocks(c, p.span, p.s, head, p.span.first + (int)(at - p.start), (int)(upto - at), lane);
        if (one_unit || p.start < at) {
            put_down();
        } else if (upto == stop) {
            Meeting m;
            m.top = w.top;
            m.total = columns_sum(w.total);
            write_row(p, m, w.acc, w.unit * (1.0f / kLift));
        } else {
            open = true;
        }
        at = upto;
        if (at == stop && at < end) next_unit(p);
    }
    if (one_unit && begin == end) {                                       // fewer blocks than wavefronts
        if (quarter == 0) {
            stats[wave][0][column] = kNone;
            stats[wave][1][column] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&sums[wave][column][16 * i + 4 * quarter]) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __syncthreads();

    // the sums of rows over this workgroup's blocks of a unit that goes on in other workgroups
    auto publish_part = [&](int which, const Meeting &m, const float (&x)[kPart]) {
        const size_t slot = 2 * (size_t)blockIdx.x + which;
#pragma unroll
        for (int d = 0; d < kPart; d += 2) put_word(space.sums + (slot * 16 + my_row) * D + my_d + d, x[d], x[d + 1]);
        if (threadIdx.x % kRowThreads == 0) put_word(space.stats + (slot * 16 + my_row) * 2, m.top, m.total);
    };
    bool first_meets = false, last_meets = false;                         // the workgroup has published its first / its last unit's sums
    Place group_last = group_first;
    if (one_unit) {
        Meeting m;
        float x[kPart];
#pragma unroll
        for (int d = 0; d < kPart; ++d) x[d] = 0.0f;
#pragma unroll
        for (int v = 0; v < kStepWaves; ++v) {
            float mine, others;
            m.add(stats[v][0][my_row], stats[v][1][my_row], mine, others);
#pragma unroll
            for (int d = 0; d < kPart; ++d) x[d] = x[d] * mine + sums[v][my_row][my_d + d] * others;
        }
        if (!begins_before && group_end == group_first.start + (uint32_t)group_first.span.blocks) {
            write_part(group_first, m, x);
            return;
        }
        publish_part(0, m, x);
        first_meets = true;
    } else {
        // A unit that began before this workgroup: its sums lie in the places of the wavefronts from the first one on.
        if (begins_before) {
            const uint32_t stop = group_first.start + (uint32_t)group_first.span.blocks;
            Meeting m;
            float x[kPart];
#pragma unroll
            for (int d = 0; d < kPart; ++d) x[d] = 0.0f;
            for (int v = 0; v < kStepWaves; ++v) {
                const uint32_t from = group_begin + group_blocks * (uint32_t)v / kStepWaves, to = group_begin + group_blocks * (uint32_t)(v + 1) / kStepWaves;
                if (from >= stop) break;
                if (from == to) continue;
                float mine, others;
                m.add(stats[v][0][my_row], stats[v][1][my_row], mine, others);
#pragma unroll
                for (int d = 0; d < kPart; ++d) x[d] = x[d] * mine + sums[v][my_row][my_d + d] * others;
            }
            publish_part(0, m, x);
            first_meets = true;
        }
        // A unit that a wavefront began and others went on with.
        if (open) {
            const uint32_t stop = p.start + (uint32_t)p.span.blocks;
            Meeting m;
            m.top = w.top;
            m.total = columns_sum(w.total);
            const float drop = w.unit * (1.0f / kLift);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) w.acc[i] *= drop;
            for (int v = wave + 1; v < kStepWaves; ++v) {
                const uint32_t from = group_begin + group_blocks * (uint32_t)v / kStepWaves, to = group_begin + group_blocks * (uint32_t)(v + 1) / kStepWaves;
                if (from >= stop) break;
                if (from == to) continue;
                float mine, others;
                m.add(stats[v][0][column], stats[v][1][column], mine, others);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) w.acc[i] = w.acc[i] * mine + *reinterpret_cast<const f32x4 *>(&sums[v][column][16 * i + 4 * quarter]) * others;
            }
            if (stop <= group_end) {
                write_row(p, m, w.acc, 1.0f);
            } else {
                const size_t slot = 2 * (size_t)blockIdx.x + 1;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) put_word(space.sums + (slot * 16 + column) * D + 16 * i + 4 * quarter + e, w.acc[i][e], w.acc[i][e + 1]);
                if (quarter == 0) put_word(space.stats + (slot * 16 + column) * 2, m.top, m.total);
            }
        }
        group_last = place_of_block(group_end - 1);
        last_meets = group_last.start + (uint32_t)group_last.span.blocks > group_end;
    }

    if (!first_meets && !last_meets) return;
    // A device-scope store has reached every XCD when it is acknowledged; the counters are raised after all threads' stores are.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    auto counter_of = [&](const Place &u) { return space.arrived + share_of(u.start); };
    if (threadIdx.x == 0) {
        if (first_meets) order[0] = __hip_atomic_fetch_add(counter_of(group_first), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (last_meets) order[1] = __hip_atomic_fetch_add(counter_of(group_last), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    auto join = [&](const Place &u, uint32_t before_me) {
        const uint32_t from = share_of(u.start), to = share_of(u.start + (uint32_t)u.span.blocks - 1);
        if (before_me != to - from) return;                               // not the last one
        if (threadIdx.x == 0) __hip_atomic_store(counter_of(u), 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        Meeting m;
        float x[kPart];
#pragma unroll
        for (int d = 0; d < kPart; ++d) x[d] = 0.0f;
        constexpr int kAhead = kPart > 4 ? 2 : 4;                         // shares whose sums are requested together
        for (uint32_t g0 = from; g0 <= to; g0 += kAhead) {
            Word y[kAhead][kPart / 2], stat[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint32_t g = g0 + j <= to ? g0 + j : to;
                const size_t slot = 2 * (size_t)g + (begin_of(g) < u.start ? 1 : 0);
                stat[j] = get_word(space.stats + (slot * 16 + my_row) * 2);
#pragma unroll
                for (int d = 0; d < kPart / 2; ++d) y[j][d] = get_word(space.sums + (slot * 16 + my_row) * D + my_d + 2 * d);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (g0 + j > to) break;
                float mine, others;
                m.add(as_float((uint32_t)stat[j]), as_float((uint32_t)(stat[j] >> 32)), mine, others);
#pragma unroll
                for (int d = 0; d < kPart / 2; ++d) {
                    x[2 * d] = x[2 * d] * mine + as_float((uint32_t)y[j][d]) * others;
                    x[2 * d + 1] = x[2 * d + 1] * mine + as_float((uint32_t)(y[j][d] >> 32)) * others;
                }
            }
        }
        write_part(u, m, x);
    };
    if (first_meets) join(group_first, order[0]);
    if (last_meets) join(group_last, order[1]);
}

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
        if (lanes_max(row.high) < block * kBlock) continue;
        f16x8 q[D / 32];
        const float back = load_queries<D, BF16>(q, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, row.high >= 0, lane);
        const float scale = a.scale * back * kLog2e * scale_k;
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
    float *weights = c.weights + weight_at(c, page, head);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = sum[t][e];
#pragma unroll
            for (int step = 1; step < 16; step *= 2) x += __shfl_xor(x, step);
            const int at = 16 * t + 4 * quarter + e;
            if (column == 0 && block * kBlock + at < length) weights[at] = a.decay == 0.0f ? x : __builtin_fmaf(a.decay, weights[at], x);
        }
}

}  // namespace

extern "C" int spqt_kv_workspace_bytes(int sequences, int rows, int q_heads, int kv_heads, int head_dim, int max_blocks, size_t *out_bytes) {
    if (!out_bytes) return SPQT_EINVAL;
    if (sequences < 1 || sequences > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || kv_heads > 16384 || q_heads < kv_heads || q_heads % kv_heads != 0 ||
        head_dim < 64 || head_dim > SPQT_KV_MAX_DIM || head_dim % 64 != 0 || max_blocks < 1 || max_blocks > 1 << 24)
        return SPQT_ESHAPE;
    const int group = q_heads / kv_heads;
    if ((int64_t)rows * group > 1 << 28) return SPQT_ESHAPE;
    // the step kernel's places and, where a call may be of that kind, the prompt kernel's, one or the other
    size_t bytes = 2 * kShares * 16 * (size_t)(head_dim + 2) * 4;
    if (is_prompt(rows, group) && prompt_bytes(head_dim) > bytes) bytes = prompt_bytes(head_dim);
    *out_bytes = kWorkspaceHead + kShares * 4 + bytes;
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
    const int tiles = (rows * a.group + 15) / 16;
    const bool prompt = is_prompt(rows, a.group);
    if (!prompt && (int64_t)cache->sequences * cache->kv_heads * tiles * cache->max_blocks > 0x7FFFFFFF) return SPQT_ESHAPE;
    Space space;
    space.arrived = (uint32_t *)((char *)workspace + kWorkspaceHead);
    space.stats = (float *)(space.arrived + kShares);
    space.sums = space.stats + 2 * kShares * 32;
    dispatch(*cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        constexpr bool B = decltype(bf16)::value;
        if (prompt) launch_prompt(*cache, a, space.stats, (hipStream_t)stream);
        else hipLaunchKernelGGL((spqt_kv_step_kernel<D, B>), dim3(kShares), dim3(step_threads(D)), 0, (hipStream_t)stream, view(*cache), a, space, cache->sequences, tiles);
        if (cache->weights)
            hipLaunchKernelGGL((spqt_kv_weigh_kernel<D, B>), dim3((cache->max_blocks + kWaves - 1) / kWaves, cache->kv_heads, cache->sequences), dim3(kThreads), 0,
                               (hipStream_t)stream, view(*cache), a);
    });
    return launched();
}
