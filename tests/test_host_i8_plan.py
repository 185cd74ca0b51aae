"""Which way an 8-bit product takes, on the CPU: csrc/i8_plan.hpp compiled with g++."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2511_04477_amd as spqt
from i8_paths import FAR, FEW, LAYER, MANY, PATHS, PROMPTS, layer_products, pitch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "i8_plan.hpp"
using namespace spqt::i8;

static Product product(int64_t rows, int64_t N, int64_t K, int gated, int64_t codes_row, int64_t weights_row, int64_t y_row) {
    Product p = {};
    p.codes_row = codes_row;
    p.weights_row = weights_row;
    p.y_row = y_row;
    p.rows = (int)rows;
    p.N = (int)N;
    p.K = (int)K;
    p.outputs = (int)(gated ? N / 2 : N);
    return p;
}
// out: rows and channels of a tile (0: without shared memory), parts, units, the bytes of the parts' sums
extern "C" void plan(int64_t rows, int64_t N, int64_t K, int gated, int64_t codes_row, int64_t weights_row, int64_t y_row, int64_t room, int64_t *out) {
    const Product p = product(rows, N, K, gated, codes_row, weights_row, y_row);
    const Plan way = plan_of(p, gated != 0, (size_t)room);
    for (int i = 0; i < 5; ++i) out[i] = 0;
    if (way.shape < 0) return;
    const Cost &s = kShapes[way.shape];
    out[0] = s.rows;
    out[1] = s.channels;
    out[2] = way.parts;
    out[3] = tiles_of(s, p, gated != 0) * way.parts;
    out[4] = way.parts > 1 ? out[3] * s.rows * s.channels * 4 : 0;
}
extern "C" int64_t sums(int64_t rows, int64_t N, int64_t K) { return (int64_t)most_sums(rows, N, K); }
"""
HEAD = 256


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    build = tmp_path_factory.mktemp("i8_plan")
    (build / "plan.cpp").write_text(SOURCE)
    lib = str(build / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-fPIC", "-shared", "-I",
                    os.path.join(ROOT, "paper_2511_04477_amd", "csrc"), str(build / "plan.cpp"), "-o", lib], check=True)
    L = ctypes.CDLL(lib)
    L.plan.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] + [ctypes.c_int64] * 4 + [ctypes.POINTER(ctypes.c_int64)]
    L.plan.restype = None
    L.sums.argtypes, L.sums.restype = [ctypes.c_int64] * 3, ctypes.c_int64
    return L


def way(rules, rows, N, K, gated=False, space=True, codes_row=None, weights_row=None, y_row=None):
    """(tile, parts, units, bytes of sums) that a call takes."""
    out = (ctypes.c_int64 * 5)()
    rules.plan(rows, N, K, int(gated), codes_row or pitch(K), weights_row or pitch(K), y_row or N, rules.sums(rows, N, K) if space else 0, out)
    return f"{out[0]}x{out[1]}" if out[0] else "few", out[2], out[3], out[4]


@pytest.mark.parametrize("gated", [False, True])
def test_the_sizes_of_the_gpu_tests_take_every_way(rules, gated):
    for (tile, kind), (rows, N, K) in PATHS.items():
        for space in (False, True):
            if kind == "parts" and not space:
                assert way(rules, rows, N, K, gated, space)[1] <= 1
                continue
            took, parts, units, _ = way(rules, rows, N, K, gated, space)
            assert took == tile and (parts > 1) == (kind == "parts"), (tile, kind, took, parts, units)
            assert {"one": units <= 256, "parts": units <= 256, "rounds": 256 < units, "long": 512 < units and K > 6 * 128}[kind], (tile, kind, units)
    for rows, N, K in FEW:
        assert way(rules, rows, N, K, gated)[0] == "few"


def test_the_layer_of_the_gpu_tests_goes_by_tiles(rules):
    for rows in PROMPTS:
        took = [way(rules, rows, N, K, gated, codes_row=-(-K // 128) * 128, weights_row=-(-K // 128) * 128) for N, K, gated in layer_products(*LAYER)]
        assert all(tile != "few" for tile, *_ in took) and took[3][1] > 1 and len({tile for tile, *_ in took}) > 1


def test_every_tile_has_every_way():
    assert {(tile, kind) for tile in ("256x256", "128x256", "128x128", "64x128") for kind in ("one", "parts", "rounds", "long")} == set(PATHS)


def sizes(n, seed):
    rng = random.Random(seed)
    for _ in range(n):
        yield tuple(int(round(2.0 ** rng.uniform(0, most))) for most in (24, 24, 16.99))


def test_sums_fit_the_workspace_that_is_asked_for(rules):
    for rows, N, K in sizes(3000, 1):
        need = spqt.spqt_i8_workspace_bytes(rows, N, K)
        assert need == (HEAD + rules.sums(rows, N, K) if rules.sums(rows, N, K) else 0)
        for gated in (False, True):
            if gated and N % 2:
                continue
            _, parts, units, sums = way(rules, rows, N, K, gated)
            assert sums <= rules.sums(rows, N, K) and (parts <= 1 or units <= 256) and units < 1 << 31
            assert way(rules, rows, N, K, gated, space=False)[1] <= 1


def test_places_within_a_tile_are_32_bits(rules):
    """Strides at the limits: what goes by tiles has its offsets under 2^32 and, of outputs, under 2^31 and the multiples the kernels make of them."""
    seen = set()
    for stride in ((1 << 23) - 128, 1 << 23, (1 << 23) + 128):
        for name in ("codes_row", "weights_row", "y_row"):
            took = way(rules, 398, 34898, 119, **{name: stride})[0]
            assert (took == "few") == (stride >= 1 << 23), (name, stride)
            seen.add(took)
    assert seen == {"few", "256x256"}
    for rows, N, K in ((398, 34898, 119), (262, 34722, 189)):
        last = ((1 << 32) - 1) // (N + 256) // 128 * 128              # the widest stride with which the up projection's last rows are within reach
        assert way(rules, rows, N, K, True, weights_row=last)[0] != "few"
        assert (N // 2 + 256) * last + pitch(K) < 1 << 32
        assert way(rules, rows, N, K, True, weights_row=last + 128)[0] == "few"
        assert way(rules, rows, N, K, False, weights_row=last + 128)[0] != "few"


def test_the_sizes_of_the_gpu_tests_reach_the_limits(rules):
    for rows, N, K, gated, codes_row, weights_row, y_row, tile in FAR:
        assert way(rules, rows, N, K, gated, False, codes_row, weights_row, y_row)[0] == tile
        assert max(rows * codes_row, N * weights_row, rows * y_row) > 1 << 31


def test_a_workspace_for_more_is_no_smaller(rules):
    """Along each of rows, N and K; 0 where K cannot be divided, and never over 64 MiB and a head."""
    size = spqt.spqt_i8_workspace_bytes
    for rows, N, K in sizes(1000, 2):
        here = size(rows, N, K)
        assert (here == 0) == (rows <= 16 or K <= 128) and here <= (64 << 20) + HEAD
        for more in ((rows + 1, N, K), (2 * rows, N, K), (rows, N + 1, K), (rows, 2 * N, K), (rows, N, K + 1), (rows, N, K + 129)):
            if more[0] <= 1 << 24 and more[1] <= 1 << 24 and more[2] <= 131071:
                assert size(*more) >= here, (rows, N, K, more)


def test_the_sizes_of_the_gpu_tests_have_many_rows(rules):
    for rows, N, K, tile in MANY:
        for gated in (False, True):
            took, _, units, _ = way(rules, rows, N, K, gated, False)
            assert took == tile and rows > 65535 * 16 and (tile == "few" or units > 17 * 256)
