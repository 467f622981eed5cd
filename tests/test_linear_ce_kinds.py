"""The sizes at which the linear layer's cross-entropy is tested on the GPU reach every tile kind in every
part of the work, as the library chooses them now: its table read from the source, the choice checked
against the workspace that the library asks for."""
import ctypes
import os

import pytest

import linear_ce_kinds as kinds
from paper_2609_10018_amd import ffi

P256 = 1 << 20
ALL = {2: ("Large", "Middle", "Deep", "Small", "Tiny"), 4: ("Middle", "Narrow", "Small", "Tiny")}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ffi.LIB_PATH):
        pytest.skip("library not built")
    return ffi.load_library()


OTHERS = [(2, 4096, 2048, 131072), (4, 1000, 384, 10007), (2, 16, 4096, 100003), (2, 256, 768, 1000),
          (2, 300000, 32, 2100), (4, 70000, 16, 4500), (2, 1, 64, 1 << 20), (4, 8192, 4096, 32000), (2, 0, 64, 10)]


@pytest.mark.parametrize("es,rows,dim,classes", kinds.CASES + OTHERS)
def test_the_library_chooses_the_same(lib, es, rows, dim, classes):
    d = ffi.LinearCE(1 if es == 2 else 0, dim, classes, rows, P256, dim, P256, dim, None, P256, None)
    n = ctypes.c_int64()
    for back in (0, 1):
        assert lib.elasto_linear_ce_workspace(d, back, ctypes.byref(n)) == 0
        assert n.value == (kinds.workspace(rows, dim, classes, es, bool(back)) if rows else 0)


def test_every_kind_is_tested_in_every_part():
    reached = set().union(*(kinds.parts_of(*c, w) for c in kinds.CASES for w in (False, True)))
    want = set()
    for es, names in ALL.items():
        for k in names:
            want |= {(es, "forward", k, False, False), (es, "dz", k, False, False)}
            for split in (False, True):
                if k != "Tiny":
                    want |= {(es, "dx", k, split, False), (es, "dw", k, split, False)}
            if k in ("Large", "Tiny"):
                want |= {(es, "both", k, (x, w), False) for x in (False, True) for w in (False, True)}
    # Rows set aside: products without the rows' bits, counts known on the device alone.
    for es, names in {2: ("Large", "Middle"), 4: ("Middle", "Narrow")}.items():
        for k in names:
            want |= {(es, p, k, s, True) for p in ("dx", "dw") for s in (False, True)}
            want |= {(es, "forward", k, False, True), (es, "dz", k, False, True)}
    want |= {(2, "both", "Large", (x, w), True) for x in (False, True) for w in (False, True)}
    want |= {(2, p, "Deep", False, True) for p in ("forward", "dz")}
    want |= {(4, "dx", "Small", True, True), (4, "dw", "Small", False, True), (4, "both", "Tiny", (False, False), True)}
    # Pieces of the classes whose dz run in different kinds.
    assert any(len({z[0] for z in kinds.plan(r, d, c, es)["dz"]}) > 1 for es, r, d, c in kinds.CASES)
    assert not want - reached, sorted(want - reached, key=str)
