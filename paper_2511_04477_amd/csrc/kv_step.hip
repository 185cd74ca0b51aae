// Attention of a few rows over the whole cache, softmax statistics of one pass (running maximum and sum).
//
// The rows that share a kv head - row i of the call and query head g of the head's group - are numbered r = i * group + g and taken 16 at a
// time.  What a lane of v_mfma_f32_16x16x32_f16 has of S^T = K Q^T, and so of P^T, is what it needs as an operand of O^T = V^T P^T, given the order in
// which a page holds the values (place_of): probabilities never leave their lane.  Codes are exact in fp16, so the products are those of the 16-bit
// queries with the codes; the scale of a block goes into its scores and into its probabilities.
//
// What bounds it: memory where the cache is long - one token over 131000 of 8 heads of 128, 268 MB of codes, 51.5 us = 5.2 TB/s over the whole call (6.2 once it streams) -
// and below that the chain of one workgroup: 1.5 us to its blocks, 3 for table, codes, products, 1 to join its wavefronts, 4 to join several workgroups: 8.3 us over 333 tokens
// of 8 heads, 14.7 over 4095 of 32 (33.6 MB).  40 sequences of 400 to 9500 tokens of 8 heads (346 MB) 74 us = 4.7 TB/s.
#include "kv_attend.hpp"
#include "kv_units.hpp"

namespace {

using namespace spqt;
using namespace spqt::kv;

// Where the sums of rows meet: two places for each workgroup, and a counter of what has come for the one unit that begins in it and goes on in others.
struct Space {
    uint32_t *head;      // of the workspace
    uint32_t *arrived;   // [kShares], all 0 between calls
    float *stats;        // [2 * kShares][16][2]: the rows' maxima and sums
    float *sums;         // [2 * kShares][16][D]
};
constexpr int kShares = 256;                              // workgroups of a launch: one per CU
static_assert(kShares * sizeof(uint32_t) <= kStepCounters, "counters");
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
template <int D, bool BF16, bool STREAM>
struct Wave {
    f16x8 q[D / 32];
    Row row;
    float scale, total;                  // (this lane's part of the row's sum)
    LevelUnits units;
    int full_low, full_high;             // every row sees the tokens from full_low to full_high
    f32x4 acc[D / 16];
    u32x4 k[4][D / 64], v[D / 16];

    __device__ __forceinline__ static u32x4 sixteen(const uint8_t *from) {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(from);
        return STREAM ? __builtin_nontemporal_load(p) : *p;
    }
    // The codes of a page; `on` 0: sixteen bytes of it over and over, for the last block's successor.
    __device__ __forceinline__ void fetch_keys(const uint8_t *page, uint32_t on, int lane) {
        const uint32_t at = (uint32_t)((lane & 15) * D + 16 * (lane >> 4)) & on, step = (uint32_t)D & on;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < D / 64; ++j) k[t][j] = sixteen(page + (at + 16 * t * step) + (on ? 64 * j : 0));
    }
    __device__ __forceinline__ void fetch_values(const uint8_t *page, uint32_t on, int lane) {
        const uint32_t at = (uint32_t)((lane & 15) * kBlock + 16 * (lane >> 4)) & on;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) v[i] = sixteen(page + at + 16 * i * kBlock);
    }
    // One block, whose codes have been fetched; the next one's are requested as soon as the registers are free.
    __device__ __forceinline__ void block(int number, float scale_k, float scale_v, const uint8_t *next, uint32_t on, int lane) {
        f32x4 p[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) p[t] = scores_of<D>(k[t], q);
        fetch_keys(next, on, lane);
        if (number * kBlock < full_low || number * kBlock + kBlock - 1 > full_high) {
            asm volatile("");                                // a branch: few blocks are masked
            const uint32_t from = (uint32_t)(number * kBlock + 4 * (lane >> 4) - row.low), seen = (uint32_t)(row.high - row.low);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (row.high < row.low || from + (uint32_t)(16 * t + e) > seen) p[t][e] = kNone;
        }
        float most = __builtin_fmaxf(p[0][0], p[0][1]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) most = __builtin_fmaxf(most, p[t][e]);
        most = columns_max(most);
        float by = scale * scale_k + 0x1p-126f;               // not 0: -inf times it is -inf
        if (scale_k != scale_k) {                            // a NaN for what is seen, none for the rest
            asm volatile("");
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[t][e] = p[t][e] == kNone ? kNone : scale_k;
            most = kNone;
            by = 1.0f;
        }
        const LevelUnits::Step step = units.see(most != kNone, most * by, __builtin_amdgcn_frexp_mantf(scale_v), (float)__builtin_amdgcn_frexp_expf(scale_v));
        total *= step.total;
        f16x8 lifted[2], rest[2];                            // what the matrix instructions get for a probability
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                f32x2 y;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(p[t][e + i], by, -step.from));
                    sum += x;
                    y[i] = x * step.lift;
                }
                const f16x2 h = __builtin_convertvector(y, f16x2);
                const f16x2 l = __builtin_convertvector(f32x2{y[0] - (float)h[0], y[1] - (float)h[1]}, f16x2);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    lifted[t / 2][4 * (t % 2) + e + i] = h[i];
                    rest[t / 2][4 * (t % 2) + e + i] = l[i];
                }
            }
        total += sum;
        if (scale_v != scale_v) {                            // only what is masked is none the less 0
            asm volatile("");
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (p[t][e] == kNone) lifted[t / 2][4 * (t % 2) + e] = rest[t / 2][4 * (t % 2) + e] = (_Float16)0.0f;
        }
        if (__ballot(step.sums != 1.0f))
#pragma unroll
            for (int i = 0; i < D / 16; ++i) acc[i] *= step.sums;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const f16x8 codes = codes_f16(u32x2{v[i][2 * u], v[i][2 * u + 1]});
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, lifted[u], acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, rest[u], acc[i], 0, 0, 0);
            }
        }
        fetch_values(next + kBlock * D, on, lane);
    }
    // The sums to units of 2^(top + kRoom).
    __device__ __forceinline__ void settle() {
        const int drop = units.drop() - kRoom;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] = __builtin_ldexpf(acc[i][e], drop);
    }
    // Blocks first .. first + n - 1 of the sequence.  Pages and scales of 64 of them are looked up at once, one per lane; the loads of the first ones go out
    // one chain after the other, the queries' among them.
    __device__ __forceinline__ void run(const Cache &c, const Call &a, const Span &span, int s, int head, int tile, int first, int n, int lane) {
        const int32_t *table = c.table + (size_t)s * c.max_blocks;
        for (int done = 0; done < n; done += 64) {
            const int b0 = first + done, here = n - done < 64 ? n - done : 64;
            uint32_t page = 0;
            const bool mine = lane < here && (b0 + lane) * kBlock < span.length;
            if (mine) page = (uint32_t)table[b0 + lane];
            u32x4 raw[D / 32];
            if (done == 0) {
                const int r = tile * 16 + (lane & 15);
                row = row_of(a, r, head, span.length, span.count);
                const bool inside = r < a.rows * a.group;
                full_low = rows_max(inside ? row.low : 0);
                full_high = rows_min(inside ? row.high : 0x7FFFFFFF);
                if (!inside) row.high = -1;
                load_queries<D>(raw, a.q.data + s * a.q.sequence + row.i * a.q.row + row.head * a.q.head, row.high >= 0, lane);
            }
            const bool there = mine && page < c.pages;
            if (!there) page = 0;
            float scales[2] = {__builtin_nanf(""), __builtin_nanf("")};
            if (there) {
                scales[0] = c.scales[scale_at(c, page, head, 0)];
                scales[1] = c.scales[scale_at(c, page, head, 1)];
            }
            auto codes_of = [&](int i) { return c.codes + codes_at(c, lane_of(page, i), head, 0); };
            auto scale_of = [&](int i, int which) { return as_float(lane_of(as_u32(scales[which]), i)); };
            const uint8_t *now = codes_of(0);
            fetch_keys(now, ~0u, lane);
            fetch_values(now + kBlock * D, ~0u, lane);
            if (done == 0) {
                scale = positive_scale(a.scale, raw) * kLog2e;
                scale *= queries_f16<BF16>(raw, q, 16);
                units.start();
                total = 0.0f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) acc[i] = {0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll 1
            for (int i = 0; i < here; ++i)
                block(b0 + i, scale_of(i, 0), scale_of(i, 1), codes_of(i + 1 < here ? i + 1 : i), i + 1 < here ? ~0u : 0u, lane);
        }
        settle();
    }
};

// Up to 16 rows of a kv head and sequence, a unit, share one pass over its blocks.  The blocks of all units are dealt out to at most 256 workgroups in one of
// three ways, which all workgroups work out from the lengths:
//   - short units, up to four blocks for each of a workgroup's wavefronts, go to a workgroup each if there is one for every unit: joining the sums of
//     several workgroups costs some 4 us, as long as a wavefront takes for several blocks;
//   - where units can be divided into even parts of at most half more than their share of a workgroup, every workgroup takes such a part
//     (131000 tokens of 8 heads 51.6 us, 57.0 in the third way; 12 sequences of 400 to 9500 tokens 32.4 and 35.3; twice to four times their share: 24 sequences 60.5 and 52.7);
//   - otherwise all units' blocks, in order, are divided evenly, so that workgroups end together whatever the lengths are.
// A workgroup's blocks are divided evenly among its wavefronts.  A unit that lies within one wavefront's share is written by it; the parts of one that lies
// within one workgroup's meet in shared memory; those of a longer one in the workspace, where the workgroup that comes last joins them, in order.
template <int D, bool BF16, bool STREAM>
__global__ __launch_bounds__(step_threads(D)) void spqt_kv_step_kernel(Cache c, Call a, Space space, int sequences, int tiles) {
    constexpr int kStepWaves = step_threads(D) / 64;
    constexpr uint32_t kLongest = 4 * kStepWaves;         // blocks of a unit that is not divided
    __shared__ float sums[kStepWaves][16][D + 4];
    __shared__ float stats[kStepWaves][2][16];
    __shared__ uint32_t order[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = lane & 15, quarter = lane >> 4;
    const uint32_t units_each = (uint32_t)(c.kv_heads * tiles);          // of a sequence
    poison_for_gemv(space.head);

    // the first 64 sequences stay in the lanes
    Span nearby = {0, 0, 0, 0};
    if (lane < sequences) nearby = span_of(c, a, lane);
    auto blocks_from = [&](int s0) { return s0 == 0 ? (uint32_t)nearby.blocks : (s0 + lane < sequences ? (uint32_t)span_of(c, a, s0 + lane).blocks : 0u); };
    uint32_t all = 0, most = 0;                           // blocks, and the longest unit's
    for (int s0 = 0; s0 < sequences; s0 += 64) {
        const uint32_t n = blocks_from(s0);
        all += lane_of(sum_upto(n), 63);
        const uint32_t longest = lane_of(over_lanes(n, [](uint32_t x, uint32_t y) { return x > y ? x : y; }), 63);
        most = longest > most ? longest : most;
    }
    all *= units_each;
    // workgroups, if each has at most this many blocks of one unit (all of it or an even part)
    auto parts_of = [&](uint32_t n, uint32_t each) { return (n + each - 1) / each; };
    auto groups_with = [&](uint32_t each) {
        uint32_t n = 0;
        for (int s0 = 0; s0 < sequences; s0 += 64) n += lane_of(sum_upto(s0 + lane < sequences ? parts_of(blocks_from(s0), each) : 0u), 63);
        return n * units_each;
    };
    uint32_t each, shares;
    bool aligned;
    if (most <= kLongest && (uint32_t)sequences * units_each <= (uint32_t)kShares && all <= kShares * kStepWaves) {
        each = most;
        shares = (uint32_t)sequences * units_each;
        aligned = true;
    } else {
        each = (all + kShares - 1) / kShares;
        if (each < kStepWaves) each = kStepWaves;
        const uint32_t limit = each + each / 2;
        do {
            shares = groups_with(each);
            aligned = shares <= (uint32_t)kShares;
            if (!aligned) each += each / 16 + 1;
        } while (!aligned && each <= limit);
    }
    // places in the order of all units: workgroups where each has blocks of one unit, blocks otherwise
    auto size_of = [&](uint32_t n) { return aligned ? parts_of(n, each) : n; };
    uint32_t more = 0;
    if (!aligned) {
        shares = all < kShares * kStepWaves ? (all + kStepWaves - 1) / kStepWaves : (uint32_t)kShares;
        each = all / shares;
        more = all % shares;                                              // so many workgroups have one block more
    }
    if (blockIdx.x >= shares) return;
    // Workgroups go to the 8 XCDs in turn: each gets a stretch of the order, so that the tiles of a head, which read the same blocks, share an L2:
    // 48 rows of each of 8 heads over 32000 tokens 32.2 us (39.7 in turn), 64 rows of each of 8 sequences of up to 4000 tokens 31.3 (42.0), 32 and 64 over 32000 24.9 and 33.1 either way.
    const uint32_t xcd = blockIdx.x % 8, place = shares / 8 * xcd + (xcd < shares % 8 ? xcd : shares % 8) + blockIdx.x / 8;
    auto begin_of = [&](uint32_t g) { return g * each + (g < more ? g : more); };
    auto share_of = [&](uint32_t block) { return block < more * (each + 1) ? block / (each + 1) : more + (block - more * (each + 1)) / each; };

    struct Place {
        Span span;
        int s;
        uint32_t unit, start;            // number among the sequence's units; its first place
    };
    auto nearby_span = [&](int s) {
        if (s >= 64) return span_of(c, a, s);
        Span v;
        v.length = (int)lane_of((uint32_t)nearby.length, s);
        v.count = (int)lane_of((uint32_t)nearby.count, s);
        v.first = (int)lane_of((uint32_t)nearby.first, s);
        v.blocks = (int)lane_of((uint32_t)nearby.blocks, s);
        return v;
    };
    // the unit that has this place
    auto find = [&](uint32_t at) {
        Place p;
        p.s = 0;
        uint32_t before = 0, in_front = 0;
        for (int s0 = 0; s0 < sequences; s0 += 64) {
            const uint32_t mine = s0 + lane < sequences ? size_of(blocks_from(s0)) * units_each : 0u, upto = sum_upto(mine);
            const uint64_t past = __ballot(before + upto > at);
            if (past) {
                const int l = (int)__builtin_ctzll(past);
                p.s = s0 + l;
                in_front = before + lane_of(upto - mine, l);
                break;
            }
            before += lane_of(upto, 63);
        }
        p.span = nearby_span(p.s);
        const uint32_t size = size_of((uint32_t)p.span.blocks);
        p.unit = (at - in_front) / size;
        p.start = in_front + p.unit * size;
        return p;
    };
    auto next_unit = [&](Place &p) {                                      // (of an even division)
        p.start += (uint32_t)p.span.blocks;
        if (++p.unit == units_each) {
            p.unit = 0;
            ++p.s;
            if (p.s < sequences) p.span = nearby_span(p.s);
        }
    };

    // this workgroup's blocks and the unit that the first one is of; those of one unit are counted from its start
    auto even_part = [](uint32_t n, uint32_t part, uint32_t parts) { return n / parts * part + (part < n % parts ? part : n % parts); };
    Place group_first;
    uint32_t group_begin, group_end, from = 0, to = 0;                    // from .. to: the workgroups of that unit, if all of this one's blocks are of it
    bool one_unit;
    if (aligned) {
        group_first = find(place);
        const uint32_t blocks = (uint32_t)group_first.span.blocks, parts = parts_of(blocks, each);
        from = group_first.start;
        to = from + parts - 1;
        group_begin = even_part(blocks, place - from, parts);
        group_end = even_part(blocks, place - from + 1, parts);
        group_first.start = 0;
        one_unit = true;
    } else {
        group_begin = begin_of(place);
        group_end = begin_of(place + 1);
        group_first = find(group_begin);
        one_unit = group_end <= group_first.start + (uint32_t)group_first.span.blocks;
    }
    const bool begins_before = group_first.start < group_begin;
    const uint32_t group_blocks = group_end - group_begin;
    auto begin_in_group = [&](int v) { return group_begin + group_blocks * (uint32_t)v / kStepWaves; };
    const uint32_t begin = begin_in_group(wave), end = begin_in_group(wave + 1);
    auto tile_of = [&](const Place &p) { return tiles == 1 ? 0 : (int)(p.unit % (uint32_t)tiles); };
    auto head_of = [&](const Place &p) { return tiles == 1 ? (int)p.unit : (int)(p.unit / (uint32_t)tiles); };

    Wave<D, BF16, STREAM> w;
    // the rows' sums so far to this wavefront's place in shared memory
    auto put_down = [&]() {
        const float total = columns_sum(w.total);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&sums[wave][column][16 * i + 4 * quarter]) = w.acc[i];
        if (quarter == 0) {
            stats[wave][0][column] = w.units.top;
            stats[wave][1][column] = total;
        }
    };
    // a lane's row of a unit, from its (whole) sums in registers
    auto write_row = [&](const Place &p, const Meeting &m, const f32x4 (&x)[D / 16]) {
        const int r = tile_of(p) * 16 + column;
        if (r >= a.rows * a.group) return;
        const int i = r / a.group, head = head_of(p) * a.group + r % a.group;
        uint16_t *out = a.out.data + p.s * a.out.sequence + i * a.out.row + head * a.out.head + 4 * quarter;
        const float by = m.inverse();
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            *reinterpret_cast<u32x2 *>(out + 16 * d) = u32x2{narrow2_within<BF16>(x[d][0] * by, x[d][1] * by), narrow2_within<BF16>(x[d][2] * by, x[d][3] * by)};
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
    auto write_part = [&](const Place &p, int row, const Meeting &m, const float (&x)[kPart]) {
        const int r = tile_of(p) * 16 + row;
        if (r >= a.rows * a.group) return;
        const int i = r / a.group, head = head_of(p) * a.group + r % a.group;
        uint16_t *out = a.out.data + p.s * a.out.sequence + i * a.out.row + head * a.out.head + my_d;
        const float by = m.inverse();
#pragma unroll
        for (int d = 0; d < kPart; d += 2) *reinterpret_cast<uint32_t *>(out + d) = narrow2_within<BF16>(x[d] * by, x[d + 1] * by);
        if (a.lse && threadIdx.x % kRowThreads == 0) a.lse[((size_t)p.s * a.rows + i) * a.q_heads + head] = m.lse();
    };
    auto live_rows = [&](const Place &p) {
        const int n = a.rows * a.group - tile_of(p) * 16;
        return n < 16 ? n : 16;
    };

    Place p = group_first;
    if (!one_unit && begin >= group_first.start + (uint32_t)group_first.span.blocks && begin < end) p = find(begin);
    bool open = false;                                                    // sums of a unit that goes on in the next wavefront are in registers
    for (uint32_t at = begin; at < end;) {
        const uint32_t stop = p.start + (uint32_t)p.span.blocks, upto = stop < end ? stop : end;
        w.run(c, a, p.span, p.s, head_of(p), tile_of(p), p.span.first + (int)(at - p.start), (int)(upto - at), lane);
        if (one_unit || p.start < at) {
            put_down();
        } else if (upto == stop) {
            Meeting m;
            m.top = w.units.top;
            m.total = columns_sum(w.total);
            write_row(p, m, w.acc);
        } else {
            open = true;
        }
        at = upto;
        if (at == stop && at < end) next_unit(p);
    }
    __syncthreads();

    // the rows' sums over this workgroup's part of its first unit, from the places of the wavefronts that have some of it
    auto meet_in_group = [&](uint32_t stop, Meeting &m, float (&x)[kPart]) {
#pragma unroll
        for (int d = 0; d < kPart; ++d) x[d] = 0.0f;
#pragma unroll
        for (int v = 0; v < kStepWaves; ++v) {
            if (begin_in_group(v) >= stop) break;
            if (begin_in_group(v) == begin_in_group(v + 1)) continue;
            float mine, others;
            m.add(stats[v][0][my_row], stats[v][1][my_row], mine, others);
#pragma unroll
            for (int d = 0; d < kPart; ++d) x[d] = x[d] * mine + sums[v][my_row][my_d + d] * others;
        }
    };
    auto publish_part = [&](const Meeting &m, const float (&x)[kPart]) {
        if (my_row >= live_rows(group_first)) return;
        const size_t slot = 2 * (size_t)place;
#pragma unroll
        for (int d = 0; d < kPart; d += 2) put_word(space.sums + (slot * 16 + my_row) * D + my_d + d, x[d], x[d + 1]);
        if (threadIdx.x % kRowThreads == 0) put_word(space.stats + (slot * 16 + my_row) * 2, m.top, m.total);
    };
    const uint32_t first_stop = group_first.start + (uint32_t)group_first.span.blocks;
    bool first_meets = begins_before || (one_unit && group_end < first_stop), last_meets = false;
    Place group_last = group_first;
    if (one_unit || begins_before) {
        Meeting m;
        float x[kPart];
        meet_in_group(first_stop, m, x);
        if (!first_meets) {
            write_part(group_first, my_row, m, x);
            return;
        }
        publish_part(m, x);
    }
    if (!one_unit) {
        // A unit that a wavefront began and others went on with.
        if (open) {
            const uint32_t stop = p.start + (uint32_t)p.span.blocks;
            Meeting m;
            m.top = w.units.top;
            m.total = columns_sum(w.total);
            for (int v = wave + 1; v < kStepWaves; ++v) {
                if (begin_in_group(v) >= stop) break;
                if (begin_in_group(v) == begin_in_group(v + 1)) continue;
                float mine, others;
                m.add(stats[v][0][column], stats[v][1][column], mine, others);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) w.acc[i] = w.acc[i] * mine + *reinterpret_cast<const f32x4 *>(&sums[v][column][16 * i + 4 * quarter]) * others;
            }
            if (stop <= group_end) {
                write_row(p, m, w.acc);
            } else if (column < live_rows(p)) {
                const size_t slot = 2 * (size_t)place + 1;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) put_word(space.sums + (slot * 16 + column) * D + 16 * i + 4 * quarter + e, w.acc[i][e], w.acc[i][e + 1]);
                if (quarter == 0) put_word(space.stats + (slot * 16 + column) * 2, m.top, m.total);
            }
        }
        group_last = find(group_end - 1);
        last_meets = group_last.start + (uint32_t)group_last.span.blocks > group_end;
    }

    if (!first_meets && !last_meets) return;
    // A device-scope store has reached every XCD when it is acknowledged; the counters are raised after all threads' stores are.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const uint32_t first_from = aligned ? from : share_of(group_first.start), last_from = aligned ? 0u : share_of(group_last.start);
    if (threadIdx.x == 0) {
        if (first_meets) order[0] = __hip_atomic_fetch_add(space.arrived + first_from, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (last_meets) order[1] = __hip_atomic_fetch_add(space.arrived + last_from, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    // The last one of workgroups from .. to joins their sums.  Threads of rows that a unit does not have take some of the workgroups' too.
    auto join = [&](const Place &u, uint32_t before_me, uint32_t from, uint32_t to) {
        if (before_me != to - from) return;
        if (threadIdx.x == 0) __hip_atomic_store(space.arrived + from, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int live = live_rows(u), rows = live > 8 ? 16 : (live > 4 ? 8 : (live > 2 ? 4 : live)), row = my_row & (rows - 1), helpers = 16 / rows;
        Meeting m;
        float x[kPart];
#pragma unroll
        for (int d = 0; d < kPart; ++d) x[d] = 0.0f;
        constexpr int kAhead = kPart > 4 ? 4 : 8;                         // workgroups whose sums are requested together
        for (uint32_t g0 = from + (uint32_t)(my_row / rows); g0 <= to; g0 += kAhead * helpers) {
            Word y[kAhead][kPart / 2], stat[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint32_t g = g0 + j * helpers <= to ? g0 + j * helpers : to;
                const size_t slot = 2 * (size_t)g + (!aligned && begin_of(g) < u.start ? 1 : 0);
                stat[j] = get_word(space.stats + (slot * 16 + row) * 2);
#pragma unroll
                for (int d = 0; d < kPart / 2; ++d) y[j][d] = get_word(space.sums + (slot * 16 + row) * D + my_d + 2 * d);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (g0 + j * helpers > to) break;
                float mine, others;
                m.add(as_float((uint32_t)stat[j]), as_float((uint32_t)(stat[j] >> 32)), mine, others);
#pragma unroll
                for (int d = 0; d < kPart / 2; ++d) {
                    x[2 * d] = x[2 * d] * mine + as_float((uint32_t)y[j][d]) * others;
                    x[2 * d + 1] = x[2 * d + 1] * mine + as_float((uint32_t)(y[j][d] >> 32)) * others;
                }
            }
        }
        if (helpers > 1) {
            __syncthreads();                                              // shared memory is free
#pragma unroll
            for (int d = 0; d < kPart; ++d) sums[0][my_row][my_d + d] = x[d];
            if (threadIdx.x % kRowThreads == 0) {
                stats[0][0][my_row] = m.top;
                stats[0][1][my_row] = m.total;
            }
            __syncthreads();
            for (int h = 1; h < helpers && my_row < rows; ++h) {
                float mine, others;
                m.add(stats[0][0][my_row + h * rows], stats[0][1][my_row + h * rows], mine, others);
#pragma unroll
                for (int d = 0; d < kPart; ++d) x[d] = x[d] * mine + sums[0][my_row + h * rows][my_d + d] * others;
            }
        }
        if (my_row < rows) write_part(u, row, m, x);
    };
    if (first_meets) join(group_first, order[0], first_from, aligned ? to : share_of(first_stop - 1));
    if (last_meets) join(group_last, order[1], last_from, share_of(group_last.start + (uint32_t)group_last.span.blocks - 1));
}

}  // namespace

namespace spqt {
namespace kv {

size_t step_bytes(int dim) { return 2 * (size_t)kShares * 16 * (dim + 2) * 4; }

bool step_fits(const spqt_kv_cache &cache, const Call &a) {
    return (int64_t)cache.sequences * cache.kv_heads * ((a.rows * a.group + 15) / 16) * cache.max_blocks <= 0x7FFFFFFF;
}

void launch_step(const spqt_kv_cache &cache, const Call &a, void *workspace, void *counters, void *space, hipStream_t stream) {
    const int tiles = (a.rows * a.group + 15) / 16;
    Space s;
    s.head = (uint32_t *)workspace;
    s.arrived = (uint32_t *)counters;
    s.stats = (float *)space;
    s.sums = s.stats + 2 * kShares * 32;
    // Codes that are read past the caches where they have room for more than half of the 256 MB cache: 131000 tokens of 70B heads 62.4 / 57.0 us, 40 sequences of up
    // to 9500 tokens of 8B heads 76.8 / 73.9; less than that may still be there from the last call, 4095 tokens of 7B heads 14.7 / 15.0, 13B drafts 22.9 / 23.7.
    // With a window, what counts are the blocks that it can reach: the drafts with windows of 2000, 1000 and 500 19.8 / 20.7, 15.1 / 16.6 and 11.8 / 12.3, of 4000 (they stream) 29.5.
    const int64_t reach = a.window > 0 ? ((int64_t)a.window + a.rows + kBlock - 2) / kBlock + 1 : cache.max_blocks, blocks = reach < cache.max_blocks ? reach : cache.max_blocks;
    const bool streams = cache.sequences * blocks * cache.kv_heads * cache.head_dim * 2 * kBlock > (int64_t)128 << 20;
    dispatch(cache, [&](auto dim, auto bf16) {
        constexpr int D = decltype(dim)::value;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(kShares), dim3(step_threads(D)), 0, stream, view(cache), a, s, cache.sequences, tiles);
        };
        if (streams) launch(spqt_kv_step_kernel<D, decltype(bf16)::value, true>);
        else launch(spqt_kv_step_kernel<D, decltype(bf16)::value, false>);
    });
}

}  // namespace kv
}  // namespace spqt
