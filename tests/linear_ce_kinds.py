"""The tile kinds that the linear layer's cross-entropy runs a call's products in, as linear_ce.hip chooses
them: its table of rounds is read from the source, its estimate is computed again in fp32."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_10018_amd", "csrc",
                      "linear_ce.hip")
F = np.float32


def _rounds():
    text = open(SOURCE).read()
    table = text[text.index("kRounds[2][5]"):]
    rows = re.findall(r"\{Kind::(\w+), (\d+), (\d+), (\d+), ([\d.]+)f, ([\d.]+)f, ([\d.]+)f\}",
                      table[:table.index(";")])
    rows = [(k, int(m), int(n), int(g), F(a), F(b), F(c)) for k, m, n, g, a, b, c in rows]
    assert len(rows) == 10
    return {2: rows[:5], 4: rows[5:]}


ROUNDS = _rounds()


def up(n, to):
    return -(-n // to) * to


def way(m, n, k, es, may_split):
    """(kind, columns of its tile, parts of K)."""
    best, least = ("Small", 64, 1), F(np.inf)
    steps = -(-k * es // 128)
    for kind, rows, cols, groups, step, alone, end in ROUNDS[es]:
        t, slots = -(-m // rows) * -(-n // cols), 256 * groups
        most = max(1, min(slots // t, steps // 8, 64)) if may_split else 1
        for parts in (most, 1):
            full, left = divmod(t * parts, slots)
            each = F(-(-steps // parts))
            us = F(full) * (step * each + end)
            if left:
                held = -(-left // 256)
                one = step if groups == 1 else alone + (step - alone) * F(held - 1) / F(groups - 1)
                us = us + (one * each + end)
            if parts > 1:
                us = us + (F(3) + F(parts * m * n) * F(8e-6) / F(4.5))
            if us < least:
                least, best = us, (kind, cols, parts)
    return best


def gathers(rows, dim, classes, es):
    return 64 <= rows <= 1 << 18 and 2.0 * rows * dim * classes * (1 if es == 2 else 8) > 4e10


def piece(rows, classes, es):
    fit = (256 << 20) // (max(1, rows) * es) // 256 * 256
    return min(up(classes, 256), max(2048, fit))


def plan(rows, dim, classes, es):
    """The ways of the forward pass, of each piece's dz, of dx and of dW."""
    p = piece(rows, classes, es)
    return dict(forward=way(rows, classes, dim, es, False),
                dz=[way(rows, min(p, classes - c), dim, es, False) for c in range(0, classes, p)],
                dx=way(rows, dim, p, es, True), dw=way(p, dim, rows, es, True), piece=p)


def _gather_bytes(rows, dim, classes, es):
    if not gathers(rows, dim, classes, es):
        return 0
    return sum(up(n, 256) for n in [4, -(-rows // 64) * 4] + [rows * 4] * 4 + [rows * dim * es])


def workspace(rows, dim, classes, es, backward):
    """Bytes, which the ways' tiles and parts go into."""
    w = plan(rows, dim, classes, es)
    if not backward:
        tiles = -(-classes // w["forward"][1])
        return up(tiles * rows * 8, 256) + up(rows * 4, 256) + _gather_bytes(rows, dim, classes, es)
    p, sizes = w["piece"], []
    sizes += [up(_gather_bytes(rows, dim, classes, es), 256), up(rows, 256) // 8, rows * p * es, -(-rows // 32) * p * 4]
    sizes += [w["dx"][2] * rows * dim * 4 if w["dx"][2] > 1 or p < classes else 0]
    sizes += [w["dw"][2] * p * dim * 4 if w["dw"][2] > 1 else 0]
    return sum(up(n, 256) for n in sizes)


# (bytes of an element, rows, dim, classes): with and without weights of rows these reach every kind in every
# part that it can take (KINDS, and the test that says so).
CASES = [
    # bf16.  Small and tiny products, in one and in several parts.
    (2, 1, 8, 3), (2, 2, 8, 1316), (2, 1750, 8, 2), (2, 362, 360, 1816), (2, 5590, 176, 2), (2, 8978, 40, 4),
    (2, 1593, 8, 1331), (2, 1, 8, 24756),
    # 128x128, two a CU and one.
    (2, 2, 8, 33200), (2, 1077, 1952, 2363), (2, 5148, 840, 1066), (2, 5480, 328, 5), (2, 3593, 2168, 2615),
    (2, 1463, 1384, 1297), (2, 4445, 1440, 267), (2, 1645, 1312, 1343), (2, 708, 976, 4665), (2, 2092, 5416, 1816),
    (2, 3498, 2648, 2251), (2, 1683, 1936, 6173),
    # 256x256, dx and dW apart and in one launch, in parts and whole, and in pieces of the classes.
    (2, 392, 1536, 5549), (2, 4323, 1160, 3443), (2, 6975, 1696, 5), (2, 1953, 3848, 2741), (2, 4885, 1200, 3606),
    (2, 2107, 4136, 2031), (2, 2373, 4376, 2020), (2, 1760, 2448, 4569), (2, 2162, 1984, 4901), (2, 4292, 2160, 2032),
    (2, 4909, 2216, 2297), (2, 5077, 952, 4979), (2, 6910, 392, 19233), (2, 5778, 2160, 1752), (2, 6521, 304, 10989),
    (2, 7952, 320, 16729),
    # fp32, 32x32 and 64x64.
    (4, 1, 4, 2), (4, 1, 4, 524), (4, 704, 4, 2), (4, 703, 4, 562), (4, 1323, 1280, 1575), (4, 5383, 656, 713),
    (4, 550, 852, 6171), (4, 1658, 744, 2365), (4, 1791, 1068, 12), (4, 6797, 140, 3), (4, 358, 680, 1684),
    (4, 34, 4, 17042), (4, 16, 2088, 258), (4, 1084, 596, 4088),
    # 128x64 and 128x128.
    (4, 1, 4, 34690), (4, 1000, 388, 10007), (4, 943, 1452, 1875), (4, 853, 1832, 1780), (4, 1881, 1032, 302),
    (4, 6567, 304, 3), (4, 2300, 1364, 840), (4, 3330, 680, 1107), (4, 386, 1084, 6144), (4, 1897, 1268, 1164),
    (4, 2, 72, 49970), (4, 8965, 648, 4), (4, 3180, 1980, 425), (4, 2484, 612, 1776), (4, 2734, 448, 2286),
    (4, 38, 4, 50707), (4, 6814, 44, 10856),
]


def parts_of(es, rows, dim, classes, weights):
    """What a call of these sizes launches: {(bytes, part, kind, in parts of K, rows set aside)}."""
    w, aside = plan(rows, dim, classes, es), weights and gathers(rows, dim, classes, es)
    out = {(es, "forward", w["forward"][0], False, aside)} | {(es, "dz", z[0], False, aside) for z in w["dz"]}
    (kx, _, nx), (kw, _, nw) = w["dx"], w["dw"]
    if kx == kw and kx in ("Large", "Tiny"):
        return out | {(es, "both", kx, (nx > 1, nw > 1), aside)}
    return out | {(es, "dx", kx, nx > 1, aside), (es, "dw", kw, nw > 1, aside)}
