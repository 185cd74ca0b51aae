// The product in 8-bit integers, a tile of rows and channels a workgroup: codes and weights go through shared memory.
//
// With the weights as its first operand v_mfma_i32_32x32x32_i8 gives a lane four channels of one row in turn, which belong next to each other in y.
// Sums of products are whole numbers under 2^31, so that neither the order of K nor its parts change a result. A workgroup goes from unit to unit (a
// tile, and a part of K) without a pause: loads of the next unit's first steps are on their way while the last one's outputs are made. Loads go past
// the registers to shared memory, a line of memory a row and step, and are waited for by their number, with one barrier a step.
//
// What bounds it: 256 x 256 tiles the power of the card. 4001 x 4096 x 14336 190 to 195 us and 8192 x 8192 x 8192 415 to 445 us = 2.4 to 2.6 POPS, by
// the card (a library's product of the latter 440 to 462); 4001 x 28672 x 4096 with the gate 384 to 414 us = 2.3 to 2.4 POPS, the clock down to 1.7 GHz, matrix units
// busy for 0.73 of the time, shared memory for 0.30, without conflicts but for the outputs. The matrix instructions alone, with the same codes, come
// to 3.5 POPS, with the reads of shared memory to 2.85. Wavefronts of 128 x 128 in place of 128 x 64 read a third less from it: 206 us for 190, the
// registers do not suffice for the outputs. 128 x 256 tiles are 0.9 as fast, 128 x 128 0.7 (with two workgroups a CU, of two and three steps' room,
// 0.78: 6396 x 8192 x 698 96 -> 74 us, where 256 x 256 takes 67). Small sizes: some 7 us of a launch, a first step's way from memory and a last
// tile's outputs, and with parts the sums' way there and back: 250 x 4096 x 14336 takes 25 to 30 us with weights that are partly in the cache behind
// memory, 23 of them this kernel's and 5.2 the join's, and 32 with weights from memory. Few rows: the weights' way from memory, 40 x 8192 x 28672 46 to 48 us of this kernel = 4.9 to 5.1 TB/s.
#ifndef SPQT_I8_TILES_HPP
#define SPQT_I8_TILES_HPP

#include "i8_gemm.hpp"

namespace spqt {
namespace i8 {

// A divisor with floor(2^32 / by), or 2^32 - 1 for 1: n times that is the quotient's 2^32 or up to n less, so that its upper half is the quotient or one less.
struct Divisor {
    uint32_t by, inverse;
};
inline Divisor divisor(uint32_t by) { return {by, by == 1 ? 0xFFFFFFFFu : (uint32_t)(((uint64_t)1 << 32) / by)}; }
__device__ __forceinline__ int divided(uint32_t n, Divisor d, int &rest) {
    uint32_t q = __umulhi(n, d.inverse), r = n - q * d.by;
    const bool more = r >= d.by;
    rest = (int)(more ? r - d.by : r);
    return (int)(more ? q + 1 : q);
}

// What a launch's workgroups do: units of a tile and a part of K each.
struct Tiling {
    int row_tiles, channel_tiles, wide;
    int tiles, parts, units;
    int steps;                           // of K
    Divisor by_tiles, by_parts, by_group, by_wide, by_last;      // by_group: tiles of `wide` row tiles; by_last: row tiles that are left behind whole groups
    i32x4 *sums;                         // of the parts, where there are several: a unit's lanes one after the other
    uint32_t *head;                      // of the workspace
};

// The unit of a workgroup in a round of kGroups, or -1. Workgroups go to the eight XCDs in turn: each of them gets neighbours, which share rows and
// channels in its cache.
__device__ __forceinline__ int unit_of(const Tiling &t, int round) {
    const int first = round * kGroups, left = t.units - first, here = left < kGroups ? left : kGroups, each = (here + 7) >> 3;
    const int in = ((int)blockIdx.x & 7) * each + ((int)blockIdx.x >> 3);
    return left > 0 && (int)blockIdx.x >> 3 < each && in < here ? first + in : -1;
}

// Which unit is which: `wide` row tiles side by side are gone through channel tile by channel tile; then the next part.
struct Unit {
    int row_tile, channel_tile, begin, end;      // steps
};
__device__ __forceinline__ Unit unit_at(const Tiling &t, int at) {
    int tile, in, rest;
    const int part = divided(at, t.by_tiles, tile), group = divided(tile, t.by_group, in);
    Unit u;
    u.channel_tile = divided(in, (group + 1) * t.wide <= t.row_tiles ? t.by_wide : t.by_last, rest);
    u.row_tile = group * t.wide + rest;
    u.begin = t.parts == 1 ? 0 : divided(t.steps * part, t.by_parts, rest);
    u.end = t.parts == 1 ? t.steps : divided(t.steps * (part + 1), t.by_parts, rest);
    return u;
}

// 16 bytes of each lane from base + offset to shared memory from `to` on, lane after lane. No register receives it: waits for it are written out.
__device__ __forceinline__ void load_to_shared(const int8_t *base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "memory");
}

// The same number, as one that is not known from before: what depends on it is worked out where it is used, since there are no registers for it in
// the loop over K.
__device__ __forceinline__ int anew(int v) {
    asm("" : "+v"(v));
    return v;
}

// TM rows by TN channels, WM by WN wavefronts of MI by NI matrix instructions' 32 by 32 each. Shared memory has room for NA steps of the rows and NB
// of the channels.
template <int TM, int TN, int WM, int WN, int NA, int NB>
struct Shape {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int kRows = TM / WM, kChannels = TN / WN, MI = kRows / 32, NI = kChannels / 32;
    static constexpr int kLoadsA = TM / (8 * kWaves), kLoadsB = TN / (8 * kWaves);
    static constexpr int kRoomA = TM * kStep, kRoomB = TN * kStep, kShared = NA * kRoomA + NB * kRoomB;
    // A wavefront alone on its SIMD, which has registers enough, reads a whole step ahead; two of them read 32 bytes of K ahead.
    static constexpr bool kAhead = kWaves == 4 && MI * NI <= 4;
    // Loads that are younger than those of the next step, where a step's wait is (turn() has the order of loads).
    static constexpr int kYounger = ((NA < NB ? NA : NB) - 2) * (kLoadsA + kLoadsB) + (NB > NA && !kAhead ? kLoadsB : 0);
    static_assert((!kAhead || NB == NA + 1) && NA >= 2 && NB >= 2 && kShared <= 160 * 1024 && kYounger < 64 && kWaves % 2 == 0 && 64 * kChannels <= kLoadsB * 1024);
};

// What becomes of the sums of 32 rows and a wavefront's channels, from channel n0 on: a lane has fours of channels of one row. They go through shared
// memory and leave 16 bytes a lane.
template <class S, int YT, bool GATED>
struct Finish {
    static constexpr int kOut = GATED ? S::kChannels / 2 : S::kChannels, kBytes = YT == SPQT_I8_FP32 ? 4 : 2;
    static constexpr int kTimes = kOut * kBytes > 128 ? kOut * kBytes / 128 : 1;       // that the channels are divided into, on their way
    struct Scales {
        f32x4 of[S::NI][4];
    };
    const Product &p;
    const int n0, line, half;
    const bool inside;
    __device__ __forceinline__ Finish(const Product &p_, int n0_, int line_, int half_) : p(p_), n0(n0_), line(line_), half(half_), inside(n0_ + kOut <= p_.outputs) {}

    // the first channel of the q-th four that this lane has in the n-th 32, and how far from there its numbers are
    __device__ __forceinline__ int channel(int n, int q) const { return n0 + (GATED && n >= S::NI / 2 ? n - S::NI / 2 : n) * 32 + q * 8 + half * 4; }
    __device__ __forceinline__ int behind(int n) const { return GATED && n >= S::NI / 2 ? p.outputs : 0; }
    __device__ __forceinline__ f32x4 four(const float *of, int n, int q) const { return *reinterpret_cast<const f32x4_at4 *>(of + (uint32_t)(behind(n) + channel(n, q))); }
    __device__ __forceinline__ f32x4 four_at_edge(const float *of, int n, int q) const {
        f32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = of[(uint32_t)(behind(n) + (channel(n, q) + e < p.outputs ? channel(n, q) + e : p.outputs - 1))];
        return r;
    }
    // Of all this lane's channels; where not all of them are `inside`, one by one.
    __device__ __forceinline__ void scales(Scales &s) const {
#pragma unroll
        for (int n = 0; n < S::NI; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) s.of[n][q] = four(p.weight_scales, n, q);
    }
    __device__ __forceinline__ void scales_at_edge(Scales &s) const {
#pragma unroll
        for (int n = 0; n < S::NI; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) s.of[n][q] = four_at_edge(p.weight_scales, n, q);
    }
    __device__ __forceinline__ float scale_of_row(int first) const { return p.scales[first + line < p.rows ? first + line : p.rows - 1]; }

    // stage: where this wavefront has kilobytes of shared memory of its own, `apart` bytes from each other
    __device__ __forceinline__ void rows(const i32x16 (&acc)[S::NI], int first, float scale, const Scales &by, uint8_t *stage, int apart, int lane) const {
        auto values = [&](int n, int q) {
#pragma clang fp contract(off)
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (float)acc[n][q * 4 + e] * scale * by.of[n][q][e];
            if (p.bias) {
                const f32x4 more = inside ? four(p.bias, n, q) : four_at_edge(p.bias, n, q);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += more[e];
            }
            return v;
        };
        constexpr int kLine = kOut * kBytes / kTimes, kSixteens = kLine / 16, kN = kOut / 32 / kTimes;            // bytes of a row on its way
        constexpr int kEach = 64 / kSixteens;                                                                     // rows an instruction
        // The 16s of a row are in an order of its own: places differ from a lane's first one in bits that do not depend on the lane.
        uint8_t *const put = stage + (line * kLine >> 10) * apart + (line * kLine & 1023);
        const int put_at = ((line ^ (kBytes == 4 ? half : 0)) & (kSixteens - 1)) * 16 + (kBytes == 4 ? 0 : half * 8);
        const int row_in = lane / kSixteens, c16 = lane % kSixteens;
        const uint8_t *const get = stage + row_in * kLine + ((c16 ^ (row_in & (kSixteens - 1))) << 4);
        static_assert(kEach * kLine == 1024 && kEach % kSixteens == 0, "an instruction reads a kilobyte, whose rows' orders are those of the first");
        const uint32_t lane_at = (uint32_t)row_in * (uint32_t)p.y_row * kBytes + c16 * 16;
#pragma unroll
        for (int part = 0; part < kTimes; ++part) {
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 v = values(part * kN + n, q);
                    if (GATED) {
                        const f32x4 u = values(part * kN + n + S::NI / 2, q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = gated_by<YT == SPQT_I8_FP32>(v[e], u[e]);
                    }
                    uint8_t *to = put + (put_at ^ ((n * 32 + q * 8) * kBytes));
                    if (YT == SPQT_I8_FP32) *reinterpret_cast<f32x4 *>(to) = v;
                    else *reinterpret_cast<u32x2 *>(to) = u32x2{narrow2<YT == SPQT_I8_BF16>(v[0], v[1]), narrow2<YT == SPQT_I8_BF16>(v[2], v[3])};
                    __builtin_amdgcn_sched_barrier(0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (its own part of shared memory: a wavefront needs no one else)
            uint8_t *base = reinterpret_cast<uint8_t *>(p.y) + ((int64_t)first * p.y_row + n0 + part * (kOut / kTimes)) * kBytes;
            const int c = n0 + part * (kOut / kTimes) + c16 * (16 / kBytes);
            const int row = first + row_in;
            if (inside) {
#pragma unroll
                for (int i = 0; i < 32 / kEach; ++i) {
                    const u32x4 out = *reinterpret_cast<const u32x4 *>(get + i * apart);
                    if (row + i * kEach < p.rows) *reinterpret_cast<u32x4_at2 *>(base + (int64_t)(i * kEach) * p.y_row * kBytes + lane_at) = out;
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < 32 / kEach; ++i) {
                    const u32x4 out = *reinterpret_cast<const u32x4 *>(get + i * apart);
                    uint8_t *to = base + (int64_t)(i * kEach) * p.y_row * kBytes + lane_at;
                    if (row + i * kEach >= p.rows) break;
#pragma unroll
                    for (int e = 0; e < 16 / kBytes; ++e) {
                        if (c + e >= p.outputs) break;
                        if (kBytes == 4) reinterpret_cast<uint32_t *>(to)[e] = out[e % 4];
                        else reinterpret_cast<uint16_t *>(to)[e] = (uint16_t)(out[e / 2] >> (16 * (e % 2)));
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
};

template <int TM, int TN, int WM, int WN, int NA, int NB, int YT, bool GATED>
__global__ __launch_bounds__(WM * WN * 64, 1) void spqt_i8_tiles_kernel(Product p, Tiling t) {
    typedef Shape<TM, TN, WM, WN, NA, NB> S;
    __shared__ __attribute__((aligned(1024))) uint8_t shared[S::kShared];
    const uint32_t shared_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int line = lane & 31, half = lane >> 5;
    constexpr int kMade = GATED ? TN / 2 : TN;                    // outputs of a row
    const bool ragged = p.K % kStep != 0;

    // Loading: eight rows an instruction, a row's 16s in an order that differs from row to row, so that 16 rows' 16s of one place of K lie in 16
    // different sets of banks.
    auto swizzle = [](int row) { return row >> 1 & 7; };
    const int row_in = lane >> 3, sixteen = (lane & 7) ^ swizzle(wave * 8 + row_in);
    // Where the loads of one operand are: a unit's step, its room in shared memory, and what the lanes' offsets are from.
    struct Cursor {
        int round, step, end, room;
        const int8_t *from;
    };
    Cursor ca = {0, 0, 0, 0, nullptr}, cb = {0, 0, 0, 0, nullptr};
    uint32_t a_off[S::kLoadsA], b_off[S::kLoadsB];
    if (unit_of(t, 0) < 0) return;
    auto aim_a = [&]() {
        const Unit u = unit_at(t, unit_of(t, ca.round));
        const int row0 = u.row_tile * TM;
        const int in = anew(row_in);
        ca.step = u.begin;
        ca.end = u.end;
        ca.from = p.codes + row0 * p.codes_row + u.begin * kStep;
#pragma unroll
        for (int i = 0; i < S::kLoadsA; ++i) {
            int r = (i * S::kWaves + wave) * 8 + in;
            r = row0 + r < p.rows ? r : p.rows - 1 - row0;
            a_off[i] = (uint32_t)r * (uint32_t)p.codes_row + sixteen * 16;
        }
    };
    auto aim_b = [&]() {
        const Unit u = unit_at(t, unit_of(t, cb.round));
        const int n0 = u.channel_tile * kMade;
        const int in8 = anew(row_in);
        cb.step = u.begin;
        cb.end = u.end;
        cb.from = p.weights + n0 * p.weights_row + u.begin * kStep;
#pragma unroll
        for (int i = 0; i < S::kLoadsB; ++i) {
            int r = (i * S::kWaves + wave) * 8 + in8;
            if (GATED) {
                // a wavefront's channels: half of them the gate's, half of them the same ones of the up projection
                const int in = r % S::kChannels, up = in >= S::kChannels / 2;
                r = r / S::kChannels * (S::kChannels / 2) + in - (up ? S::kChannels / 2 : 0);
                r = (n0 + r < p.outputs ? r : p.outputs - 1 - n0) + (up ? p.outputs : 0);
            } else {
                r = n0 + r < p.N ? r : p.N - 1 - n0;
            }
            b_off[i] = (uint32_t)r * (uint32_t)p.weights_row + sixteen * 16;
        }
    };
    auto load_a = [&](int i) { load_to_shared(ca.from, a_off[i], shared_at + ca.room * S::kRoomA + (i * S::kWaves + wave) * 1024); };
    auto load_b = [&](int i) { load_to_shared(cb.from, b_off[i], shared_at + NA * S::kRoomA + cb.room * S::kRoomB + (i * S::kWaves + wave) * 1024); };
    // On to the next step or tile; behind the last one the same again, which no one reads.
    // The last step of a ragged K: what lies behind the row's end is read from the step's beginning, and masked.
    auto folded = [&](const Cursor &c, auto &offsets) {
        const uint32_t back = ragged && c.step == t.steps - 1 && c.step * kStep + sixteen * 16 >= p.K ? sixteen * 16 : 0;
#pragma unroll
        for (uint32_t &o : offsets) o -= back;
    };
    auto advance = [&](Cursor &c, auto aim, auto &offsets, int rooms, auto inner) {
        c.room = c.room + 1 < rooms ? c.room + 1 : 0;
        if (decltype(inner)::value || c.step + 1 < c.end) {
            ++c.step;
            c.from += kStep;
        } else {
            if (unit_of(t, c.round + 1) < 0) return;
            ++c.round;
            aim();
        }
        if (!decltype(inner)::value) folded(c, offsets);
    };
    auto advance_a = [&](auto inner) { advance(ca, aim_a, a_off, NA, inner); };
    auto advance_b = [&](auto inner) { advance(cb, aim_b, b_off, NB, inner); };
    const std::false_type no;
    const std::true_type yes;

    // Multiplying: of the 32s of K in a step, lanes 0 to 31 have the first 16 of a 32 and the others the second.
    i32x16 acc[S::MI][S::NI];
    constexpr int kSets = S::kAhead ? 8 : 2, kReads = S::MI + S::NI, kProducts = S::MI * S::NI;
    i32x4 x[kSets][S::MI], w[kSets][S::NI];                       // of 32s of K
    int place[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) place[kk] = line * kStep + (((kk * 2 + half) ^ swizzle(line)) << 4);
    int room_a = 0, room_b = 0, next_a = 0, next_b = 0;           // of this step and the next one
    auto read = [&](bool next, int kk, int set, int i) {
        if (i < S::NI) w[set][i] = *reinterpret_cast<const i32x4 *>(shared + NA * S::kRoomA + (next ? next_b : room_b) * S::kRoomB + place[kk] + (wn * S::kChannels + i * 32) * kStep);
        else x[set][i - S::NI] = *reinterpret_cast<const i32x4 *>(shared + (next ? next_a : room_a) * S::kRoomA + place[kk] + (wm * S::kRows + (i - S::NI) * 32) * kStep);
    };
    auto mask = [&](int kk, int set, int step, auto tail) {
        if (decltype(tail)::value && ragged && step == t.steps - 1)
#pragma unroll
            for (int i = 0; i < S::MI; ++i) x[set][i] = masked(x[set][i], step * kStep + (kk * 2 + half) * 16, p.K);
    };
    auto product = [&](int set, int i) {
        const int m = i / S::NI, n = i % S::NI;
        acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[set][n], x[set][m], acc[m][n], 0, 0, 0);
    };
    auto multiply = [&](auto kk_, int step, auto tail) {
        constexpr int kk = decltype(kk_)::value, kPer = (kReads + kProducts - 1) / kProducts;
        mask(kk, kk & 1, step, tail);
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            product(kk & 1, i);
#pragma unroll
            for (int j = i * kPer; j < (i + 1) * kPer && j < kReads; ++j)
                if (kk < 3 || !decltype(tail)::value) read(kk == 3, (kk + 1) % 4, (kk + 1) & 1, j);
            if (kk == 3) {
#pragma unroll
                for (int j = 0; j < S::kLoadsA; ++j)
                    if (j * kProducts / S::kLoadsA == i) load_a(j);
            } else {
#pragma unroll
                for (int j = 0; j < S::kLoadsB; ++j)
                    if (j * 3 * kProducts / S::kLoadsB == kk * kProducts + i) load_b(j);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Until the next step's loads are there, of all wavefronts; younger ones may be on their way.
    auto meet = [&](auto younger) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(decltype(younger)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, S::kYounger> Younger;
    // inner: a step in the middle of a unit, from which both cursors move on to the next step and no other; tail: the last one of a unit.
    auto turn = [&](int step, auto odd_, auto inner, auto tail) {
        next_a = room_a + 1 < NA ? room_a + 1 : 0;
        next_b = room_b + 1 < NB ? room_b + 1 : 0;
        if constexpr (S::kAhead) {
            // Step t is in registers, everyone's; B(t - 1 + NB), A(t + NA) are loaded and step t + 1 read beside its products.
            constexpr int kOdd = decltype(odd_)::value, kAll = 4 * kProducts, kLoads = S::kLoadsA + S::kLoadsB, kPer = (4 * kReads + kAll - 1) / kAll;
            meet(Younger());
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mask(kk, 4 * kOdd + kk, step, tail);
#pragma unroll
            for (int i = 0; i < kAll; ++i) {
                product(4 * kOdd + i / kProducts, i % kProducts);
#pragma unroll
                for (int j = i * kPer; j < (i + 1) * kPer && j < 4 * kReads; ++j)
                    if (!decltype(tail)::value) read(true, j / kReads, 4 * (1 - kOdd) + j / kReads, j % kReads);
#pragma unroll
                for (int j = 0; j < kLoads; ++j)
                    if (j * kAll / kLoads == i) {
                        if (j < S::kLoadsB) load_b(j);
                        else load_a(j - S::kLoadsB);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            advance_b(inner);
            advance_a(inner);
        } else {
            // Step t: B(t - 1 + NB) is loaded beside its first three 32s of K, where step t - 1 has left room; then A(t + NA) beside the fourth, for
            // which everyone has read step t.
            multiply(std::integral_constant<int, 0>(), step, tail);
            multiply(std::integral_constant<int, 1>(), step, tail);
            multiply(std::integral_constant<int, 2>(), step, tail);
            advance_b(inner);
            meet(Younger());
            multiply(std::integral_constant<int, 3>(), step, tail);
            advance_a(inner);
        }
        room_a = next_a;
        room_b = next_b;
    };

    // the loads that the turns before the first one would have made
    aim_a();
    aim_b();
    folded(ca, a_off);
    folded(cb, b_off);
    auto all_a = [&]() {
#pragma unroll
        for (int i = 0; i < S::kLoadsA; ++i) load_a(i);
        advance_a(no);
    };
    auto all_b = [&]() {
#pragma unroll
        for (int i = 0; i < S::kLoadsB; ++i) load_b(i);
        advance_b(no);
    };
    if constexpr (S::kAhead) {
#pragma unroll 1
        for (int j = 0; j < NA; ++j) {
            all_b();
            all_a();
        }
        meet(std::integral_constant<int, (NA - 1) * (S::kLoadsA + S::kLoadsB)>());
    } else {
#pragma unroll 1
        for (int j = -(NA > NB ? NA : NB); j < -1; ++j) {
            if (j + NA >= 0) all_a();
            if (j + NB >= 0) all_b();
        }
        meet(Younger());
        all_a();
    }

    for (int round = 0;; ++round) {
        const int at = unit_of(t, round);
        if (at < 0) break;
        const Unit u = unit_at(t, at);
        const int row0 = u.row_tile * TM + wm * S::kRows;
#pragma unroll
        for (int m = 0; m < S::MI; ++m)
#pragma unroll
            for (int n = 0; n < S::NI; ++n) acc[m][n] = i32x16{};
        // (a unit's first operands are read here, the others beside the products before them: what is read after a unit's outputs needs no registers
        // while these are made)
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, 1> odd;
#pragma unroll
        for (int kk = 0; kk < kSets / 2; ++kk)
#pragma unroll
            for (int i = 0; i < kReads; ++i) read(false, kk, kk, i);
        int s = u.begin;
        const int inner = u.end - (NA > NB ? NA : NB) - 2;
        if constexpr (S::kAhead) {
            for (; s + 1 < inner; s += 2) {
                turn(s, even, yes, no);
                turn(s + 1, odd, yes, no);
            }
            for (; s + 2 < u.end; s += 2) {
                turn(s, even, no, no);
                turn(s + 1, odd, no, no);
            }
        } else {
            for (; s < inner; ++s) turn(s, even, yes, no);
            for (; s < u.end - 1; ++s) turn(s, even, no, no);
        }
        const int here = anew(lane);
        const Finish<S, YT, GATED> finish(p, u.channel_tile * kMade + wn * (S::kChannels / (GATED ? 2 : 1)), here & 31, here >> 5);
        // Asked for before the last step, used after it. A load that no one waited for would make the compiler wait in the next unit's loop, for the
        // loads that are on their way there.
        typename Finish<S, YT, GATED>::Scales by;
        float scales[S::MI];
        if (t.parts == 1 && finish.inside) finish.scales(by);
        if (t.parts == 1)
#pragma unroll
            for (int m = 0; m < S::MI; ++m) scales[m] = finish.scale_of_row(row0 + m * 32);
        if (S::kAhead && s + 1 < u.end) {
            turn(s, even, no, no);
            turn(s + 1, odd, no, yes);
        } else {
            turn(s, even, no, yes);
        }

        if (t.parts > 1) {
            i32x4 *to = t.sums + ((size_t)at * S::kWaves + wave) * (S::MI * S::NI * 256);
#pragma unroll
            for (int m = 0; m < S::MI; ++m)
#pragma unroll
                for (int n = 0; n < S::NI; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        (to + ((m * S::NI + n) * 4 + q) * 64)[here] = i32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                        __builtin_amdgcn_sched_barrier(0);
                    }
            continue;
        }
        if (!finish.inside) finish.scales_at_edge(by);
        // The last step's room of the channels is free until the next turn: outputs go through what this wavefront's own loads will write there.
        uint8_t *stage = shared + NA * S::kRoomA + (room_b > 0 ? room_b - 1 : NB - 1) * S::kRoomB + wave * 1024;
#pragma unroll
        for (int m = 0; m < S::MI; ++m) {
            const int again = anew(lane);
            Finish<S, YT, GATED>(p, finish.n0, again & 31, again >> 5).rows(acc[m], row0 + m * 32, scales[m], by, stage, S::kWaves * 1024, again);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // no load may arrive after the workgroup has left its shared memory
}

// The parts' sums together, and what becomes of them: a workgroup takes 32 rows of what a wavefront of the other kernel had, each of its four
// wavefronts every fourth part.
template <int TM, int TN, int WM, int WN, int NA, int NB, int YT, bool GATED>
__global__ __launch_bounds__(256) void spqt_i8_join_kernel(Product p, Tiling t) {
    typedef Shape<TM, TN, WM, WN, NA, NB> S;
    __shared__ __attribute__((aligned(1024))) uint8_t stage[S::kLoadsB * 1024];
    __shared__ i32x4 sums[3][S::NI * 4][64];
    const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), line = lane & 31, half = lane >> 5;
    const int m = blockIdx.x % S::MI, wave = blockIdx.x / S::MI % S::kWaves, tile = blockIdx.x / (S::MI * S::kWaves);
    if (blockIdx.x == 0 && threadIdx.x == 0) *t.head = 1u;         // (a GEMV on this workspace is to yield NaN)
    const Unit u = unit_at(t, tile);
    const Finish<S, YT, GATED> finish(p, u.channel_tile * (GATED ? TN / 2 : TN) + wave % WN * (S::kChannels / (GATED ? 2 : 1)), line, half);
    const int first = u.row_tile * TM + wave / WN * S::kRows + m * 32;
    if (first >= p.rows) return;
    typename Finish<S, YT, GATED>::Scales by;                     // asked for beside the sums
    float scale = 0.0f;
    if (own == 0) {
        if (finish.inside) finish.scales(by);
        else finish.scales_at_edge(by);
        scale = finish.scale_of_row(first);
    }
    i32x16 acc[S::NI];
#pragma unroll
    for (int n = 0; n < S::NI; ++n) acc[n] = i32x16{};
    auto add = [&](const i32x4 *from) {
#pragma unroll
        for (int n = 0; n < S::NI; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const i32x4 v = from[(n * 4 + q) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][4 * q + e] += v[e];
            }
    };
#pragma unroll 2
    for (int part = own; part < t.parts; part += 4) add(t.sums + ((((size_t)part * t.tiles + tile) * S::kWaves + wave) * S::MI + m) * S::NI * 256 + lane);
    if (own > 0)
#pragma unroll
        for (int n = 0; n < S::NI; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) sums[own - 1][n * 4 + q][lane] = i32x4{acc[n][4 * q], acc[n][4 * q + 1], acc[n][4 * q + 2], acc[n][4 * q + 3]};
    __syncthreads();
    if (own > 0) return;
#pragma unroll
    for (int i = 0; i < 3; ++i) add(&sums[i][0][lane]);
    finish.rows(acc, first, scale, by, stage, 1024, lane);
}

template <int TM, int TN, int WM, int WN, int NA, int NB, int YT, bool GATED>
void launch_tiles_as(const Product &p, const Tiling &t, hipStream_t stream) {
    typedef Shape<TM, TN, WM, WN, NA, NB> S;
    const int grid = t.units < kGroups ? (t.units + 7) / 8 * 8 : kGroups;
    hipLaunchKernelGGL((spqt_i8_tiles_kernel<TM, TN, WM, WN, NA, NB, YT, GATED>), dim3(grid), dim3(S::kThreads), 0, stream, p, t);
    if (t.parts > 1)
        hipLaunchKernelGGL((spqt_i8_join_kernel<TM, TN, WM, WN, NA, NB, YT, GATED>), dim3(t.tiles * S::kWaves * S::MI), dim3(256), 0, stream, p, t);
}

// In `parts` parts of K, whose sums take parts * tiles * TM * TN * 4 bytes from 256 bytes behind the workspace's beginning on.
template <int TM, int TN, int WM, int WN, int NA, int NB>
void launch_tiles(const Product &p, bool gated, int parts, void *workspace, hipStream_t stream) {
    const int made = gated ? TN / 2 : TN;
    Tiling t;
    t.row_tiles = (p.rows + TM - 1) / TM;
    t.channel_tiles = (p.outputs + made - 1) / made;
    t.wide = t.row_tiles < 8 ? t.row_tiles : 8;
    t.tiles = t.row_tiles * t.channel_tiles;
    t.parts = parts;
    t.units = t.tiles * parts;
    t.steps = (p.K + kStep - 1) / kStep;
    t.by_tiles = divisor(t.tiles);
    t.by_parts = divisor(parts);
    t.by_group = divisor(t.wide * t.channel_tiles);
    t.by_wide = divisor(t.wide);
    t.by_last = divisor(t.row_tiles % t.wide > 0 ? t.row_tiles % t.wide : t.wide);
    t.head = (uint32_t *)workspace;
    t.sums = (i32x4 *)((uint8_t *)workspace + kWorkspaceHead);
    auto typed = [&](auto yt) {
        if (gated) launch_tiles_as<TM, TN, WM, WN, NA, NB, decltype(yt)::value, true>(p, t, stream);
        else launch_tiles_as<TM, TN, WM, WN, NA, NB, decltype(yt)::value, false>(p, t, stream);
    };
    if (p.y_type == SPQT_I8_FP32) typed(std::integral_constant<int, SPQT_I8_FP32>());
    else if (p.y_type == SPQT_I8_BF16) typed(std::integral_constant<int, SPQT_I8_BF16>());
    else typed(std::integral_constant<int, SPQT_I8_FP16>());
}

}  // namespace i8
}  // namespace spqt
#endif
