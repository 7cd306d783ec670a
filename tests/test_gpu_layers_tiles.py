"""Every tile shape of the layers' matrix-core products, in each form, for one and two halves,
with the sum split and whole, against the definition in 64 bits.

The tables below hold ragged shapes (m, k, n) for each: odd m, and k and n odd (16-bit operands
are copied to aligned rows) or multiples of 8 (read in place), sums of one and two stages of 64
among them.  Which tile a shape takes is asked of the library's own planner.

Tolerances.  A sum of L terms in fp32, whose signs are random, is off by up to 25 sqrt(L) E times
the root mean square of the results (E = 2^-23; each addition is off by half an ulp of a partial
sum of a few times that; the 6 products of fp32 parts count as 6 L).  What goes into the
gradients' products is exact: relu's slopes, and factors that are powers of two.  The result is
rounded to u of it, half a unit in the last place of its type.
"""

import ctypes
import math

import pytest
import torch

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {name: torch.finfo(t).eps / 2 for name, t in DT.items()}
TINY = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -25, "fp32": 2.0 ** -149}
E = 2.0 ** -23
CUS = 256
TILES = 4

# (operands, form, halves, tile, sum split, shapes)
PRODUCTS = [
    ("16", "forward", 1, 0, False, [(3857, 259, 3231), (5251, 264, 2392)]),
    ("16", "forward", 1, 1, False, [(1861, 775, 1057), (1549, 792, 1320)]),
    ("16", "forward", 1, 1, True, [(1807, 1873, 645), (695, 3128, 920)]),
    ("16", "forward", 1, 2, False, [(5007, 29, 1163), (1425, 67, 4231), (4883, 147, 1187), (3277, 144, 1808)]),
    ("16", "forward", 1, 2, True, [(1491, 2871, 1307), (1495, 2904, 1288)]),
    ("16", "forward", 1, 3, False, [(75, 129, 21), (67, 136, 24)]),
    ("16", "forward", 1, 3, True, [(71, 513, 21), (71, 536, 24)]),
    ("16", "forward", 2, 0, False, [(2777, 257, 2205), (2275, 264, 2712)]),
    ("16", "forward", 2, 0, True, [(1545, 2821, 1299), (461, 3040, 4280)]),
    ("16", "forward", 2, 1, False, [(1419, 779, 711), (641, 832, 1496)]),
    ("16", "forward", 2, 1, True, [(603, 3077, 513), (495, 3160, 648)]),
    ("16", "forward", 2, 2, False, [(4497, 21, 647), (3503, 69, 839), (1053, 135, 2883), (2209, 152, 1360)]),
    ("16", "forward", 2, 2, True, [(867, 2841, 1169), (601, 2952, 1616)]),
    ("16", "forward", 2, 3, False, [(75, 129, 21), (67, 136, 24)]),
    ("16", "forward", 2, 3, True, [(71, 513, 21), (71, 536, 24)]),
    ("16", "dx", 1, 0, False, [(2501, 4963, 263), (4199, 2976, 264)]),
    ("16", "dx", 1, 1, False, [(1867, 1031, 825), (1629, 1168, 832)]),
    ("16", "dx", 1, 1, True, [(787, 793, 3101), (899, 648, 3112)]),
    ("16", "dx", 1, 2, False, [(5525, 1025, 31), (5461, 1035, 77), (4437, 1285, 133), (3523, 1680, 160)]),
    ("16", "dx", 1, 2, True, [(1631, 1175, 2833), (1895, 1048, 2856)]),
    ("16", "dx", 1, 3, False, [(311, 21, 215), (253, 24, 264)]),
    ("16", "dx", 1, 3, True, [(119, 23, 557), (121, 24, 552)]),
    ("16", "dx", 2, 0, False, [(3531, 2329, 455), (4199, 1936, 456)]),
    ("16", "dx", 2, 0, True, [(3649, 1097, 1495), (5469, 656, 1296)]),
    ("16", "dx", 2, 1, False, [(2307, 775, 399), (1415, 1440, 392)]),
    ("16", "dx", 2, 1, True, [(903, 665, 1615), (595, 1056, 1552)]),
    ("16", "dx", 2, 2, False, [(5525, 1025, 31), (5461, 1035, 77), (4901, 1176, 96)]),
    ("16", "dx", 2, 2, True, [(2307, 819, 1305), (1605, 1216, 1384)]),
    ("16", "dx", 2, 3, False, [(579, 21, 117), (517, 24, 128)]),
    ("16", "dx", 2, 3, True, [(119, 23, 557), (121, 24, 552)]),
    ("16", "dw", 1, 0, False, [(263, 2777, 4447), (267, 2312, 5288)]),
    ("16", "dw", 1, 1, False, [(823, 1359, 1421), (799, 2360, 784)]),
    ("16", "dw", 1, 1, True, [(2357, 1185, 775), (3177, 1136, 568)]),
    ("16", "dw", 1, 2, False, [(83, 5541, 1037), (161, 4895, 1157), (129, 3848, 1552)]),
    ("16", "dw", 1, 2, True, [(2849, 1629, 1249), (2965, 2448, 808)]),
    ("16", "dw", 1, 3, False, [(311, 21, 215), (253, 24, 264)]),
    ("16", "dw", 1, 3, True, [(571, 21, 123), (517, 24, 128)]),
    ("16", "dw", 2, 0, False, [(261, 2659, 2389), (261, 1232, 4904)]),
    ("16", "dw", 2, 0, True, [(2879, 2555, 783), (2833, 4152, 456)]),
    ("16", "dw", 2, 1, False, [(781, 1363, 757), (777, 912, 1096)]),
    ("16", "dw", 2, 1, True, [(2339, 613, 791), (3177, 616, 528)]),
    ("16", "dw", 2, 2, False, [(67, 1165, 2563), (131, 2907, 1035), (135, 1224, 2488)]),
    ("16", "dw", 2, 2, True, [(2835, 1107, 923), (2845, 1192, 856)]),
    ("16", "dw", 2, 3, False, [(311, 21, 215), (253, 24, 264)]),
    ("16", "dw", 2, 3, True, [(571, 21, 123), (517, 24, 128)]),
    ("fp32", "forward", 1, 0, False, [(1475, 21, 4097), (3713, 67, 1381), (1171, 211, 3431), (1565, 216, 2592)]),
    ("fp32", "forward", 1, 0, True, [(1357, 5329, 75), (971, 1153, 1309), (527, 1800, 1200)]),
    ("fp32", "forward", 1, 1, False, [(2121, 453, 967), (783, 456, 2520)]),
    ("fp32", "forward", 1, 1, True, [(641, 941, 1105), (843, 656, 1160)]),
    ("fp32", "forward", 1, 2, False, [(1349, 21, 2185), (2215, 65, 1363), (1053, 135, 2883), (2209, 152, 1360)]),
    ("fp32", "forward", 1, 2, True, [(389, 711, 1189), (773, 715, 915), (905, 712, 792)]),
    ("fp32", "forward", 1, 3, False, [(67, 145, 23), (67, 136, 24)]),
    ("fp32", "forward", 1, 3, True, [(71, 513, 21), (69, 576, 24)]),
    ("fp32", "forward", 2, 0, False, [(1217, 25, 2449), (833, 69, 2921), (643, 197, 3005), (707, 224, 2736)]),
    ("fp32", "forward", 2, 0, True, [(2827, 2741, 39), (523, 971, 1173), (541, 1824, 632)]),
    ("fp32", "forward", 2, 1, False, [(901, 195, 1661), (1569, 208, 984)]),
    ("fp32", "forward", 2, 1, True, [(651, 959, 555), (389, 904, 920)]),
    ("fp32", "forward", 2, 2, False, [(257, 23, 5269), (1395, 65, 1099), (961, 129, 1567), (465, 136, 3088)]),
    ("fp32", "forward", 2, 2, True, [(227, 1011, 781), (513, 739, 747), (389, 752, 872)]),
    ("fp32", "forward", 2, 3, False, [(67, 145, 23), (67, 136, 24)]),
    ("fp32", "forward", 2, 3, True, [(71, 513, 21), (69, 576, 24)]),
    ("fp32", "dx", 1, 0, False, [(5127, 1191, 29), (1309, 3905, 73), (1707, 2399, 199), (1613, 2504, 208)]),
    ("fp32", "dx", 1, 0, True, [(1375, 75, 5143), (1349, 903, 1005), (753, 920, 1864)]),
    ("fp32", "dx", 1, 1, False, [(2737, 719, 451), (1077, 2000, 456)]),
    ("fp32", "dx", 1, 1, True, [(947, 791, 935), (1155, 704, 904)]),
    ("fp32", "dx", 1, 2, False, [(3481, 837, 27), (5539, 529, 65), (2345, 1287, 131), (1461, 2120, 136)]),
    ("fp32", "dx", 1, 2, True, [(1161, 389, 711), (707, 669, 1091), (1033, 712, 752)]),
    ("fp32", "dx", 1, 3, False, [(215, 23, 313), (253, 24, 264)]),
    ("fp32", "dx", 1, 3, True, [(125, 21, 545), (127, 24, 552)]),
    ("fp32", "dx", 2, 0, False, [(4639, 1089, 25), (3405, 1169, 85), (2563, 1576, 72)]),
    ("fp32", "dx", 2, 0, True, [(1799, 129, 1405), (527, 1199, 939), (1167, 520, 936)]),
    ("fp32", "dx", 2, 1, False, [(2511, 795, 203), (1101, 1800, 216)]),
    ("fp32", "dx", 2, 1, True, [(803, 605, 641), (643, 544, 928)]),
    ("fp32", "dx", 2, 2, False, [(3481, 837, 27), (4613, 783, 89), (5431, 648, 88)]),
    ("fp32", "dx", 2, 2, True, [(649, 517, 465), (771, 589, 539), (659, 720, 544)]),
    ("fp32", "dx", 2, 3, False, [(579, 21, 117), (517, 24, 128)]),
    ("fp32", "dx", 2, 3, True, [(125, 21, 545), (127, 24, 552)]),
    ("fp32", "dw", 1, 0, False, [(75, 3909, 1293), (197, 3389, 1227), (203, 1560, 2584)]),
    ("fp32", "dw", 1, 0, True, [(5447, 133, 897), (1801, 727, 923), (1899, 640, 1120)]),
    ("fp32", "dw", 1, 1, False, [(507, 1669, 1209), (471, 1568, 1336)]),
    ("fp32", "dw", 1, 1, True, [(697, 775, 1233), (907, 672, 1216)]),
    ("fp32", "dw", 1, 2, False, [(75, 2695, 1099), (157, 2181, 1367), (135, 1224, 2488)]),
    ("fp32", "dw", 1, 2, True, [(971, 539, 649), (707, 669, 1091), (717, 1376, 560)]),
    ("fp32", "dw", 1, 3, False, [(193, 25, 341), (253, 24, 264)]),
    ("fp32", "dw", 1, 3, True, [(575, 21, 123), (517, 24, 128)]),
    ("fp32", "dw", 2, 0, False, [(71, 773, 3183), (199, 1089, 1869), (197, 904, 2264)]),
    ("fp32", "dw", 2, 0, True, [(2827, 2741, 39), (1823, 571, 585), (1955, 528, 584)]),
    ("fp32", "dw", 2, 1, False, [(205, 1089, 1371), (479, 656, 1488)]),
    ("fp32", "dw", 2, 1, True, [(1393, 579, 385), (711, 608, 824)]),
    ("fp32", "dw", 2, 2, False, [(71, 843, 1775), (129, 1217, 1273), (149, 784, 1904)]),
    ("fp32", "dw", 2, 2, True, [(723, 609, 385), (711, 533, 735), (1145, 392, 592)]),
    ("fp32", "dw", 2, 3, False, [(193, 25, 341), (253, 24, 264)]),
    ("fp32", "dw", 2, 3, True, [(575, 21, 123), (517, 24, 128)]),
]
# dx and dW of a dense (1) or gated (2) layer by one launch of a tile shape, or (-1) by two;
# neither, either or both sums split: (operands, halves, tile, shapes)
PAIRS = [
    ("16", 1, -1, [(807, 4121, 3077), (809, 4120, 3080)]),
    ("16", 1, 1, [(799, 1171, 787), (849, 1152, 936), (1581, 795, 805), (1659, 832, 776), (779, 521, 2357),
        (779, 480, 2336), (2679, 285, 1677), (2431, 152, 2464)]),
    ("16", 1, 2, [(691, 5825, 263), (303, 5912, 648), (4717, 909, 23), (3649, 1192, 24), (67, 4109, 1107),
        (75, 1936, 2368), (4337, 211, 2821), (4575, 200, 2944)]),
    ("16", 1, 3, [(311, 21, 215), (517, 24, 128), (757, 23, 87), (687, 24, 96), (95, 23, 695), (91, 24, 744),
        (1203, 27, 657), (1163, 24, 648)]),
    ("16", 2, -1, [(769, 4821, 1345), (745, 5000, 1232)]),
    ("16", 2, 1, [(901, 1037, 459), (909, 1032, 472), (2599, 397, 403), (2611, 400, 408), (791, 527, 1155),
        (823, 544, 1160), (2657, 147, 1335), (1695, 272, 1344)]),
    ("16", 2, 2, [(275, 5823, 327), (275, 5920, 344), (4717, 909, 23), (2977, 1312, 80), (71, 923, 2453),
        (69, 984, 2408), (4373, 203, 1457), (5183, 136, 1360)]),
    ("16", 2, 3, [(311, 21, 215), (253, 24, 264), (757, 23, 87), (783, 24, 88), (163, 27, 405), (185, 24, 360),
        (667, 25, 605), (673, 24, 616)]),
    ("fp32", 1, -1, [(877, 4599, 445), (821, 1432, 2728)]),
    ("fp32", 1, 0, [(429, 4749, 395), (391, 4808, 448), (1957, 1219, 149), (3869, 624, 152), (139, 2225, 1235),
        (137, 2904, 920), (1347, 363, 1347), (1359, 352, 1376)]),
    ("fp32", 1, 1, [(503, 2175, 451), (479, 2168, 504), (1161, 1133, 251), (1305, 1000, 272), (199, 1685, 805),
        (209, 1096, 1192), (1293, 321, 911), (819, 216, 1808)]),
    ("fp32", 1, 2, [(275, 5543, 261), (281, 5392, 296), (1537, 777, 157), (791, 1624, 144), (135, 1551, 791),
        (147, 1104, 1224), (983, 353, 709), (717, 136, 1488)]),
    ("fp32", 1, 3, [(193, 25, 341), (253, 24, 264), (579, 21, 117), (517, 24, 128), (95, 23, 695), (147, 32, 456),
        (467, 25, 721), (475, 32, 728)]),
    ("fp32", 2, -1, [(261, 897, 3435), (325, 1192, 2704)]),
    ("fp32", 2, 0, [(461, 4749, 197), (475, 4392, 232), (2119, 1231, 103), (2055, 1160, 128), (135, 1551, 791),
        (131, 1032, 1328), (1477, 325, 649), (1413, 352, 712)]),
    ("fp32", 2, 1, [(449, 2243, 223), (463, 2296, 200), (787, 1713, 111), (771, 1672, 104), (193, 535, 1215),
        (197, 888, 784), (909, 211, 773), (825, 200, 912)]),
    ("fp32", 2, 2, [(289, 4825, 229), (267, 4640, 296), (1057, 1235, 97), (4105, 272, 120), (79, 213, 3115),
        (95, 776, 984), (1475, 137, 331), (727, 152, 728)]),
    ("fp32", 2, 3, [(417, 21, 163), (379, 24, 176), (579, 21, 117), (517, 24, 128), (163, 27, 405), (253, 24, 264),
        (707, 31, 201), (713, 32, 208)]),
]


@pytest.fixture(scope="module")
def pid():
    from paper_2009_04509_amd import binding
    return binding


@pytest.fixture(scope="module")
def layers(pid):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    h = pid.pointid_layers_create(0)
    yield h
    h.close()


class Plan(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int), ("splits", ctypes.c_int)]


class PairPlan(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int), ("dx_splits", ctypes.c_int), ("dw_splits", ctypes.c_int)]


def plan_product(pid, f32, form, halves, m, k, n):
    """(tile, sum split) of pointid::plan_product."""
    rows, cols, h, inner, terms = {"forward": (m, n, halves, k, 1), "dx": (m, k, 1, n, halves),
                                   "dw": (k, n, halves, m, 1)}[form]
    f = pid.lib["_ZN7pointid12plan_productEbllilii"]
    i64, i32 = ctypes.c_int64, ctypes.c_int
    f.restype, f.argtypes = Plan, [ctypes.c_bool, i64, i64, i32, i64, i32, i32]
    p = f(f32, rows, cols, h, inner, terms, CUS)
    return p.tile, p.splits > 1


def plan_pair(pid, f32, halves, m, k, n):
    f = pid.lib["_ZN7pointid9plan_pairEbllliii"]
    i64, i32 = ctypes.c_int64, ctypes.c_int
    f.restype, f.argtypes = PairPlan, [ctypes.c_bool, i64, i64, i64, i32, i32, i32]
    p = f(f32, m, k, n, halves, 1, CUS)
    return p.tile, p.dx_splits > 1, p.dw_splits > 1


def test_the_tables_name_every_tile(pid):
    """The planner gives each shape the tile it stands under, and every tile is there in every
    form (16-bit pairs of 256 x 256 are not built; no cheap sum of a single half is split there)."""
    seen = set()
    for kind, form, halves, tile, split, shapes in PRODUCTS:
        for s in shapes:
            assert plan_product(pid, kind == "fp32", form, halves, *s) == (tile, split), (kind, form, halves, s)
        seen.add((kind, form, halves, tile, split))
    for kind in ("16", "fp32"):
        for form in ("forward", "dx", "dw"):
            for halves in (1, 2):
                for tile in range(TILES):
                    assert (kind, form, halves, tile, False) in seen
                    assert (kind, form, halves, tile, True) in seen or (kind, halves, tile) == ("16", 1, 0)
    for kind, halves, tile, shapes in PAIRS:
        plans = [plan_pair(pid, kind == "fp32", halves, *s) for s in shapes]
        assert {p[0] for p in plans} == {tile}
        if tile >= 0:
            assert {p[1:] for p in plans} == {(a, b) for a in (False, True) for b in (False, True)}
    assert {p[:3] for p in PAIRS} == {(kind, halves, tile) for kind in ("16", "fp32") for halves in (1, 2)
                                      for tile in range(-1, TILES)} - {("16", 1, 0), ("16", 2, 0)}


# ---- on the device

def near(got, want, tol, dtype, what):
    bad = ~((got.double() - want).abs() <= tol + want.abs() * U[dtype] + TINY[dtype])
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. at {at}: "
                             f"{got[tuple(at)].item()} for {want[tuple(at)].item()}")


def product(a, b, dtype, terms=1):
    """(a b, the bound of its fp32 error)"""
    want = a @ b
    count = terms * a.shape[1] * (6 if dtype == "fp32" else 1) + 8
    return want, 25 * math.sqrt(count) * E * want.square().mean().sqrt()


class Draw:
    def __init__(self, dtype, seed):
        self.dtype, self.g = DT[dtype], torch.Generator(device=DEV).manual_seed(seed)

    def normal(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g, device=DEV) * scale).to(self.dtype)

    def floats(self, n):
        return torch.randn(n, generator=self.g, device=DEV)

    def powers(self, *shape):
        """1, 2 and 4 with either sign"""
        e = torch.randint(0, 3, shape, generator=self.g, device=DEV)
        s = torch.randint(0, 2, shape, generator=self.g, device=DEV) * 2 - 1
        return torch.ldexp(s.float(), e).to(self.dtype)


def kept(pid, v, eight):
    """(what is handed over, its values in 64 bits)"""
    if not eight:
        return v, v.double()
    c = pid.pointid_checkpoint_save(v)
    return c, pid.pointid_checkpoint_load(c, torch.float32).double()


def near_codes(pid, c, want, tol, what):
    """A checkpoint's values: 4 significant bits, and the smallest step of its block."""
    got = pid.pointid_checkpoint_load(c, torch.float32).double()
    step = torch.ldexp(torch.ones_like(want), (c.exponents.int() - 127 - 9)[:, torch.arange(want.shape[1], device=DEV) // 32])
    bad = ~((got - want).abs() <= want.abs() / 16 * 1.01 + step + tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. at {bad.nonzero()[0].tolist()}"


def rows(table, types=("bf16", "fp16", "fp32")):
    return [pytest.param(dtype, *row[1:], id="-".join([dtype] + [str(v) for v in row[1:-1]])) for row in table
            for dtype in types if (dtype == "fp32") == (row[0] == "fp32")]


def check_forward(pid, layers, dtype, halves, m, k, n, eight):
    d = Draw(dtype, m + k + n)
    x, w = d.normal(m, k), [d.normal(k, n, scale=k ** -0.5) for _ in range(halves)]
    b = [d.floats(n) for _ in range(halves)]
    z, tz = [], []
    for i in range(halves):
        want, tol = product(x.double(), w[i].double(), dtype)
        z.append(want + b[i].double())
        tz.append(tol + z[i].abs() * 2 * E)
    save = [pid.Checkpoint.empty(m, n, DEV) if eight else torch.empty((m, n), dtype=DT[dtype], device=DEV)
            for _ in range(halves)]
    # an activation's slope is at most 1.13, and it is computed to 3e-7 of max(1, |z|)
    if halves == 1:
        r = d.normal(m, n)
        y = pid.pointid_dense(layers, x, w[0], b[0], "gelu", r, save=save[0])
        want = z[0] * torch.special.ndtr(z[0]) + r.double()
        tol = 1.13 * tz[0] + 3e-7 * z[0].abs().clamp(min=1) + want.abs() * E
    else:
        y = pid.pointid_gated(layers, x, w[0], w[1], b[0], b[1], "silu", save_g=save[0], save_u=save[1])
        a = z[0] * torch.sigmoid(z[0])
        want = a * z[1]
        ta = 1.13 * tz[0] + 3e-7 * z[0].abs().clamp(min=1)
        tol = a.abs() * tz[1] + (z[1].abs() + tz[1]) * ta + want.abs() * E
    near(y, want, tol, dtype, f"y {m} x {k} x {n}")
    for i in range(halves):
        if eight:
            near_codes(pid, save[i], z[i], tz[i], f"codes {i} {m} x {k} x {n}")
        else:
            near(save[i], z[i], tz[i], dtype, f"kept {i} {m} x {k} x {n}")


def check_backward(pid, layers, dtype, halves, m, k, n, eight, need_dx, need_dw):
    d = Draw(dtype, m + k + n + 1)
    dy = d.powers(m, n)
    w = [d.normal(k, n, scale=k ** -0.5) for _ in range(halves)]
    x, x64 = kept(pid, d.normal(m, k), eight)
    z = [kept(pid, d.normal(m, n), eight) for _ in range(halves)]
    on = (z[0][1] > 0).double()
    need_db = need_dx and need_dw
    if halves == 1:
        dz = [dy.double() * on]
        dx, *dw = pid.pointid_dense_backward(layers, dy, x, w[0], z[0][0], "relu", need_dx, need_dw, need_db)
        dw, db = dw[:1], dw[1:]
    else:
        dz = [dy.double() * z[1][1] * on, dy.double() * z[0][1] * on]
        dx, *dw = pid.pointid_gated_backward(layers, dy, x, w[0], w[1], z[0][0], z[1][0], "relu", need_dx, need_dw, need_db)
        dw, db = dw[:2], dw[2:]
    assert all(torch.equal(v.to(DT[dtype]).double(), v) for v in dz)
    if need_dx:
        want, tol = product(torch.cat(dz, 1), torch.cat([v.double().t() for v in w], 0), dtype)
        near(dx, want, tol, dtype, f"dx {m} x {k} x {n}")
    for i in range(halves):
        if need_dw:
            want, tol = product(x64.t(), dz[i], dtype)
            near(dw[i], want, tol, dtype, f"dW {i} {m} x {k} x {n}")
        if need_db:
            tol = dz[i].abs().sum(0) * (m + 2) * E
            assert ((db[i].double() - dz[i].sum(0)).abs() <= tol).all(), f"db {i} {m} x {k} x {n}"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, form, halves, tile, split, shapes", rows(PRODUCTS))
def test_products(pid, layers, dtype, form, halves, tile, split, shapes):
    for m, k, n in shapes:
        for eight in (False, True):
            if form == "forward":
                check_forward(pid, layers, dtype, halves, m, k, n, eight)
            else:
                check_backward(pid, layers, dtype, halves, m, k, n, eight, form == "dx", form == "dw")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, halves, tile, shapes", rows(PAIRS))
def test_pairs(pid, layers, dtype, halves, tile, shapes):
    for m, k, n in shapes:
        for eight in (False, True):
            check_backward(pid, layers, dtype, halves, m, k, n, eight, True, True)
