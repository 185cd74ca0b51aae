// Which kernel a product in 8-bit integers takes, and how it divides the work: plain C++, whose rules a CPU can test.
#ifndef SPQT_I8_PLAN_HPP
#define SPQT_I8_PLAN_HPP

#include <stddef.h>
#include <stdint.h>

namespace spqt {
namespace i8 {

struct Product {
    const int8_t *codes, *weights;
    const float *scales, *weight_scales, *bias;
    void *y;
    int64_t codes_row, weights_row, y_row;
    int rows, N, K;
    int outputs;             // of a row: N, gated N / 2
    int y_type;
};

constexpr int kStep = 128;               // bytes of K that a tile takes at a time: a line of memory
constexpr int kGroups = 256;             // workgroups of a launch of tiles, at most: one a CU
constexpr int kFewRows = 16;             // that always go without shared memory
constexpr int kMostParts = 16;           // of K

// A shape of tiles and the parts that K is divided into, and what that is expected to take. shape -1: without shared memory.
struct Plan {
    int shape, parts;
    double us;
};

// Bytes for the sums of a call's parts, at most. As much for larger numbers as for smaller ones, at least: a workspace for more serves less.
inline size_t most_sums(int64_t rows, int64_t N, int64_t K) {
    const int64_t steps = (K + kStep - 1) / kStep, parts = steps < kMostParts ? steps : kMostParts;
    if (rows <= kFewRows || parts == 1) return 0;
    const int64_t sums = ((rows + 63) / 64) * ((N + 127) / 128) * parts * (64 * 128 * 4), most = (int64_t)64 << 20;
    return (size_t)(sums < most ? sums : most);
}

// Of more than sixteen rows, in us: an instruction reads 16 rows, each a line of its own, which takes a CU as many cycles: 35 KB a us, of codes and
// weights alike; not before the weights are read, and 3 for the launch. Measured / this: 64 x 4096 x 4096 12.7 / 12.4, 128 x 4096 x 4096 21.7 / 21.7,
// 32 x 12288 x 4096 21.2 / 19.9, 300 x 520 x 2000 6.9 / 7.6.
inline double few_us(const Product &p, bool gated) {
    const int R = p.rows <= 32 ? 2 : 4;
    const int64_t groups = (int64_t)((p.outputs + 15) / 16) * ((p.rows + 16 * R - 1) / (16 * R));
    const double turns = (double)((groups + 255) / 256), weights = p.N * (double)p.K / 4.7e6;
    const double read = turns * ((p.rows < 16 * R ? p.rows : 16 * R) + (gated ? 32 : 16)) * p.K / 35e3;
    return 3.0 + (read > weights ? read : weights);
}

// What a shape takes, in us: a step of a lone workgroup and of one of 256, and a tile's beginning and end; and how many times as long steps are of
// rows that begin within a line, of weights that the caches do not keep. From 30 sizes of 20 to 8000 rows, 520 to 28672 channels, K of 400 to 28672;
// a step of 128 is 0.87, 0.43, 0.22 and 0.11 us of matrix instructions at 2.4 GHz. 256 of the large tiles draw so much power that the clock falls to 1.75 GHz.
struct Cost {
    int rows, channels;
    float step, step_full, fixed, within;
};
constexpr Cost kShapes[] = {
    {256, 256, 0.95f, 1.62f, 2.5f, 1.35f}, {128, 256, 0.55f, 0.93f, 2.5f, 1.5f}, {128, 128, 0.30f, 0.57f, 2.5f, 1.45f}, {64, 128, 0.22f, 0.36f, 2.0f, 1.7f}};
constexpr int kCount = sizeof(kShapes) / sizeof(kShapes[0]);

inline int64_t tiles_of(const Cost &s, const Product &p, bool gated) {
    const int made = gated ? s.channels / 2 : s.channels;
    return (int64_t)((p.rows + s.rows - 1) / s.rows) * ((p.outputs + made - 1) / made);
}

// The one that is expected to be done first:
//   - rounds of 256 workgroups, a tile's steps each;
//   - with parts, 3 us for the second launch and a us for every 3.5 MB of sums;
//   - where one tile has all rows and the weights are more than the caches keep, no sooner than 4.7 MB of weights a us, and 33 KB a us for a workgroup;
//   - steps of rows that begin within a line are in two lines: `within` times as long, a quarter where the caches keep the weights.
// Rows within lines: 270 x 11008 x 12800 / 12801 with 256 x 256 in two parts 83 / 105 us, 128 x 256 80 / 122, 128 x 128 100 / 138, 64 x 128 84 / 127;
// weights in caches: 777 x 1111 x 5003 in rows of 5120 / 5008 bytes 20.0 / 24.6. One size stands for all here: 17 x 8839 x 26019 took 67 us before and takes 69 to 71 by this rule.
// Rows x channels x K, us of 256 x 256 / 128 x 256 / 128 x 128 / 64 x 128 with the best number of parts each (the one taken is the least, or within 7 % of it):
//   4001 x 4096 x 14336   188 / 210 / 268 / 343        1500 x 5120 x 5120   52.0 / 43.1 / 49.4 / 64.0      1024 x 4096 x 4096   38.2 / 28.5 / 24.2 / 31.1
//   1024 x 8192 x 28672   207 (2 parts; one 283) / 211 / 276 / 386       250 x 4096 x 14336    36.8 (10) / 33.2 (7) / 32.3 (4; two 42.5) / 35.5 (2)
//   512 x 4096 x 4096     29.4 (3) / 25.3 / 19.3 / 17.1                  40 x 8192 x 28672    - / - / - / 50.4 (4; three, which are taken, 52.0; two 63.6, one 103)
inline Plan plan_tiles(const Product &p, bool gated, size_t room) {
    // places within a tile, with the gate's and the up projection's channels in one, are 32 bits
    const int64_t widest = (int64_t)1 << 23;
    Plan best = {-1, 1, 0.0};
    if (p.codes_row >= widest || p.weights_row >= widest || p.y_row >= widest || (gated && (p.N + 256) * p.weights_row >= (int64_t)1 << 32)) return best;
    const int steps = (p.K + kStep - 1) / kStep;
    const bool within = p.codes_row % kStep != 0 || p.weights_row % kStep != 0;
    for (int i = 0; i < kCount; ++i) {
        const Cost &s = kShapes[i];
        const int64_t tiles = tiles_of(s, p, gated);
        if (tiles > 1 << 28) continue;
        for (int parts = 1; parts == 1 || (parts <= kMostParts && parts <= steps && tiles * parts <= kGroups); ++parts) {
            const int64_t units = tiles * parts, sums = units * s.rows * s.channels * 4;
            if (parts > 1 && (size_t)sums > room) break;
            const double weights = p.N * (double)p.K, each = (steps + parts - 1) / parts * (!within ? 1.0 : weights > 20e6 ? s.within : 1.25);
            const bool streams = p.rows <= s.rows && weights > 20e6;
            auto round = [&](int64_t n) {
                const double full = s.step + (s.step_full - s.step) * (double)n / kGroups, slowest = streams ? s.channels * (128 / 33e3) : 0.0;
                return n == 0 ? 0.0 : each * (full > slowest ? full : slowest) + s.fixed;
            };
            double us = (double)(units / kGroups) * round(kGroups) + round(units % kGroups);
            if (streams && us < weights / 4.7e6) us = weights / 4.7e6;
            if (parts > 1) us += 3.0 + (double)sums / 3.5e6;
            us += 5.0;                               // the launch, and a first tile's first operands
            if (best.shape < 0 || us < best.us) best = {i, parts, us};
        }
    }
    return best;
}

// The way that a call takes with this room for sums.
inline Plan plan_of(const Product &p, bool gated, size_t room) {
    const Plan none = {-1, 1, 0.0};
    if (p.rows <= kFewRows) return none;
    const Plan tiles = plan_tiles(p, gated, room);
    return tiles.shape >= 0 && tiles.us < few_us(p, gated) ? tiles : none;
}

}  // namespace i8
}  // namespace spqt
#endif
