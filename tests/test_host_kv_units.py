"""The units of attention's running sums, on the CPU: csrc/kv_units.hpp compiled with g++, over blocks of value scales of any size, in fp32 against 64 bits."""
import ctypes
import math
import os
import random
import subprocess

import pytest

import paper_2511_04477_amd as spqt  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "kv_units.hpp"
using namespace spqt::kv;

static auto see(BlockUnits &u, bool sees, float most, float part, float exponent) { return u.see(sees, most, part, 1.0f / part, exponent); }
static auto see(LevelUnits &u, bool sees, float most, float part, float exponent) { return u.see(sees, most, part, exponent); }
static float part_of(const BlockUnits &u) { return u.part; }
static float part_of(const LevelUnits &) { return 1.0f; }
static float probability(const BlockUnits::Step &step, float score, float &number) { return (number = exp2f(score - step.less)) * step.back; }
static float probability(const LevelUnits::Step &step, float score, float &number) {
    const float p = exp2f(score - step.from);
    number = p * step.lift;
    return p;
}

// One row over `blocks` blocks of n tokens each: scores in powers of two, one code a token, a scale a block, `sees` 0 for a block that the row does not see.
// result: out in fp32, the largest number of a token, the largest sum on the way.
template <class U>
static void go(int blocks, int n, const float *scores, const float *codes, const float *scales, const int *sees, float *result) {
    U units;
    units.start();
    float acc = 0.0f, total = 0.0f, lifted = 0.0f, largest = 0.0f;
    for (int b = 0; b < blocks; ++b) {
        int exponent;
        const float part = frexpf(scales[b], &exponent);
        float most = -__builtin_inff();
        for (int t = 0; t < n; ++t) most = fmaxf(most, scores[b * n + t]);
        const auto step = see(units, sees[b] != 0, most, part, (float)exponent);
        acc *= step.sums;
        total *= step.total;
        for (int t = 0; t < n && sees[b]; ++t) {
            float y;
            total += probability(step, scores[b * n + t], y);
            acc += y * codes[b * n + t];
            lifted = fmaxf(lifted, y);
            largest = fmaxf(largest, fabsf(acc));
        }
    }
    result[0] = ldexpf(acc * part_of(units), units.drop() - 32) * (0x1p32f / (total == 0.0f ? 1.0f : total));
    result[1] = lifted;
    result[2] = largest;
}
extern "C" void by_block(int blocks, int n, const float *scores, const float *codes, const float *scales, const int *sees, float *result) {
    go<BlockUnits>(blocks, n, scores, codes, scales, sees, result);
}
extern "C" void by_level(int blocks, int n, const float *scores, const float *codes, const float *scales, const int *sees, float *result) {
    go<LevelUnits>(blocks, n, scores, codes, scales, sees, result);
}
"""


@pytest.fixture(scope="module", params=["by_block", "by_level"])
def row(request, tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2511_04477_amd", "csrc"), "-o", str(d / "units.so"), str(d / "units.cpp")], check=True)
    function = getattr(ctypes.CDLL(str(d / "units.so")), request.param)

    def call(blocks):
        """blocks: (scores, codes, scale, sees); what the row is in fp32 and in 64 bits, and how far apart they may be."""
        n = len(blocks[0][0])
        floats = lambda values: (ctypes.c_float * len(values))(*values)  # noqa: E731
        result = floats([0.0] * 3)
        scales = floats([b[2] for b in blocks])
        function(len(blocks), n, floats([x for b in blocks for x in b[0]]), floats([x for b in blocks for x in b[1]]), scales,
                 (ctypes.c_int * len(blocks))(*[int(b[3]) for b in blocks]), result)
        terms = [(s, c * scale) for (scores, codes, _, sees), scale in zip(blocks, scales) if sees for s, c in zip(scores, codes)]
        top = max((s for s, _ in terms), default=0.0)
        total = math.fsum(2.0 ** (s - top) for s, _ in terms) or 1.0
        want = math.fsum(2.0 ** (s - top) * v for s, v in terms) / total
        spread = math.fsum(2.0 ** (s - top) * abs(v) for s, v in terms) / total
        # sums of that many terms and factors of a few roundings each, twice (both sums)
        bound = spread * 2 * (len(terms) + len(blocks) + 16) * 2.0 ** -24 + 2.0 ** -149
        assert result[1] <= 2.0 ** 15 and math.isfinite(result[2])
        return result[0], want, bound
    return call


def even(sizes, n=64):
    """Blocks of equal scores with values of these sizes; a block of zeros has the least scale that there is."""
    return [([0.0] * n, [127.0 if x else 0.0] * n, max(x / 127.0, 2.0 ** -100), True) for x in sizes]


@pytest.mark.parametrize("sizes", [[8.0] * 40 + [0.0], [1.0] * 140 + [0.0] + [1.0] * 4, [1000.0, 0.0], [1.0] * 200 + [0.0] + [1.0] * 5, [4.0] * 40 + [0.0] + [4.0] * 5,
                                   [16.0] * 20 + [0.0] + [16.0] * 5, [0.0], [0.0, 3.0], [3e38, 0.0, 1e-30, 3e38], [1e-38, 65504.0, 1e-30] * 10, [1e30, 1e-30, 1.0, 1e20] * 7])
def test_blocks_of_any_size_after_one_another(row, sizes):
    got, want, bound = row(even(sizes))
    assert abs(got - want) <= bound, (got, want, bound)


def test_random_blocks(row):
    r = random.Random(5)
    for _ in range(300):
        n = r.choice([1, 3, 64])
        blocks = []
        for _ in range(r.randint(1, 40)):
            middle = r.randint(-60, 30)
            # eighths: a score less a whole number is exact
            scores = [middle + r.randint(-40, 40) / 8 for _ in range(n)]
            blocks.append((scores, [float(r.randint(-127, 127)) for _ in range(n)], math.ldexp(r.uniform(0.5, 1.0), r.randint(-99, 110)), r.random() < 0.8))
        got, want, bound = row(blocks)
        assert abs(got - want) <= bound, (got, want, bound)


def test_a_row_that_sees_nothing(row):
    assert row([([5.0], [3.0], 1.0, False), ([1.0], [3.0], 2.0 ** -100, False)]) == (0.0, 0.0, 2.0 ** -149)


def test_no_number_reaches_the_rows_that_see_it(row):
    nan = float("nan")
    for blocks in ([([0.0], [1.0], nan, True)], [([0.0], [1.0], 1.0, True), ([-90.0], [0.0], nan, True), ([3.0], [1.0], 1.0, True)]):
        assert math.isnan(row(blocks)[0])
    got, want, bound = row([([0.0], [1.0], 1.0, True), ([-9.0], [0.0], nan, False), ([3.0], [2.0], 1.0, True)])
    assert abs(got - want) <= bound
