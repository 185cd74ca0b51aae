"""Sizes of 8-bit products that take every way through the kernels, gated or not, with rows of codes and weights that begin at multiples of 16 bytes.

"one": a tile to a workgroup, at most; "parts": K is divided, and the sums are joined (with a workspace); "rounds": workgroups go on to further tiles; "long": more than twice,
with many steps each.  tests/test_host_i8_plan.py holds them to that.
"""

# (tile, way): (rows, N, K), each with edges in every dimension; the K of "rounds" is a step of 128 or two, or several.
PATHS = {
    ("256x256", "one"): (131, 33770, 247), ("256x256", "parts"): (132, 17224, 5410), ("256x256", "rounds"): (398, 34898, 119),
    ("128x256", "one"): (77, 32868, 249), ("128x256", "parts"): (271, 3988, 6971), ("128x256", "rounds"): (262, 34722, 189),
    ("128x128", "one"): (65, 21084, 372), ("128x128", "parts"): (65, 1556, 13336), ("128x128", "rounds"): (8373, 856, 1207),
    ("256x256", "long"): (2585, 12600, 898), ("128x256", "long"): (1039, 15378, 1065), ("128x128", "long"): (8410, 1834, 1420), ("64x128", "long"): (67, 49062, 3194),
    ("64x128", "one"): (461, 1054, 1278), ("64x128", "parts"): (55, 62, 3919), ("64x128", "rounds"): (150, 16708, 2290),
}
# Without shared memory: up to 16 rows, up to 32, more.
FEW = [(1, 40, 300), (15, 66, 1000), (29, 130, 700), (70, 94, 333)]


def pitch(K):
    return -(-K // 16) * 16


# A layer (hidden, heads, kv heads, dim, inner) and prompts whose products go by tiles, the last one in parts. Rows of codes begin at multiples of 128 bytes there.
LAYER = (2048, 16, 4, 128, 5632)
PROMPTS = [200, 150]


def layer_products(hidden, heads, kv_heads, dim, inner):
    """(N, K, gated) of a layer's products."""
    return [((heads + 2 * kv_heads) * dim, hidden, False), (hidden, heads * dim, False), (2 * inner, hidden, True), (hidden, inner, False)]

# Rows as far apart as tiles take them, whose places pass 2^31: (rows, N, K, gated, strides of codes, weights and y, tile). The last of each pair of gated ones is just too far for tiles.
_FAR = (1 << 23) - 128


def _reach(N):
    return ((1 << 32) - 1) // (N + 256) // 128 * 128


FAR = [
    (398, 34898, 119, False, _FAR, 128, _FAR, "256x256"), (461, 1054, 1278, False, _FAR, _FAR, _FAR, "64x128"),
    (398, 34898, 119, True, 128, _reach(34898), _FAR, "256x256"), (398, 34898, 119, True, 128, _reach(34898) + 128, 17449, "few"),
    (262, 34722, 189, True, _FAR, _reach(34722), 34722, "128x256"), (461, 1054, 1278, True, _FAR, _FAR, _FAR, "few"),
]

# More rows than one launch without shared memory takes (1048560), and tiles that go on 17 times and more.
MANY = [(1048579, 24, 40, "few"), (2100003, 16, 16, "few"), (1048579, 40, 700, "128x128"), (1048579, 300, 130, "256x256")]
