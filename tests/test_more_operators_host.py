"""Refusals of the operators of a training step, before any pointer is used or any
HIP call is made: through the C ABI with addresses that nothing may touch."""
import ctypes
import math
import os

import pytest

from paper_2609_10018_amd import ffi

P256 = 1 << 20
INVALID = 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ffi.LIB_PATH):
        pytest.skip("library not built")
    return ffi.load_library()


# ------------------------------------------------- cross-entropy of a linear layer

def ce(**kw):
    d = dict(dtype=1, dim=64, classes=1000, rows=100, x=P256, ldx=64, weight=P256, ldw=64, bias=None,
             labels=P256, row_weight=None)
    d.update(kw)
    return ffi.LinearCE(*[d[n] for n, _ in ffi.LinearCE._fields_])


CE_BAD = [dict(dtype=2), dict(dim=0), dict(dim=4), dict(dim=60), dict(dim=-8), dict(dim=(1 << 20) + 8),
          dict(classes=0), dict(classes=-1), dict(classes=(1 << 30) + 1), dict(rows=-1),
          dict(rows=(1 << 24) + 1), dict(rows=1 << 24, classes=1 << 20), dict(x=None), dict(weight=None),
          dict(labels=None), dict(x=P256 + 8), dict(weight=P256 + 2), dict(ldx=56), dict(ldw=56),
          dict(ldx=68), dict(ldw=-64), dict(ldx=1 << 21), dict(bias=P256 + 2), dict(labels=P256 + 1),
          dict(row_weight=P256 + 2), dict(dtype=0, dim=6), dict(dtype=0, ldx=66)]


@pytest.mark.parametrize("kw", CE_BAD)
def test_linear_ce_refuses_bad_descriptions(lib, kw):
    big = 1 << 45
    assert lib.elasto_op_linear_ce(ce(**kw), P256, P256, P256, big, None) == INVALID
    assert lib.elasto_op_linear_ce_bwd(ce(**kw), P256, 1.0, P256, 64, P256, 64, None, P256, big,
                                       None) == INVALID
    assert lib.elasto_last_error()


def test_linear_ce_refuses_bad_results_and_workspaces(lib):
    n = ctypes.c_int64()
    for back in (0, 1):
        assert lib.elasto_linear_ce_workspace(ce(), back, ctypes.byref(n)) == 0 and n.value > 0
        assert lib.elasto_linear_ce_workspace(ce(), back, None) == INVALID
        assert lib.elasto_linear_ce_workspace(None, back, ctypes.byref(n)) == INVALID
        assert lib.elasto_linear_ce_workspace(ce(dtype=7), back, ctypes.byref(n)) == INVALID
    big = 1 << 45
    assert lib.elasto_op_linear_ce(None, P256, P256, P256, big, None) == INVALID
    for loss, lse in ((None, P256), (P256 + 2, P256), (P256, P256 + 1)):
        assert lib.elasto_op_linear_ce(ce(), loss, lse, P256, big, None) == INVALID
    assert lib.elasto_linear_ce_workspace(ce(), 0, ctypes.byref(n)) == 0
    for ws, size in ((None, big), (P256 + 16, big), (P256, n.value - 1), (P256, -1)):
        assert lib.elasto_op_linear_ce(ce(), P256, P256, ws, size, None) == INVALID
    assert lib.elasto_linear_ce_workspace(ce(), 1, ctypes.byref(n)) == 0

    def back(lse=P256, scale=1.0, dx=P256, lddx=64, dw=P256, lddw=64, db=None, ws=P256, size=big):
        return lib.elasto_op_linear_ce_bwd(ce(), lse, scale, dx, lddx, dw, lddw, db, ws, size, None)

    for kw in (dict(lse=None), dict(lse=P256 + 2), dict(scale=math.nan), dict(scale=math.inf),
               dict(dx=P256 + 8), dict(lddx=56), dict(lddx=1 << 21), dict(dw=P256 + 4), dict(lddw=68),
               dict(db=P256 + 2), dict(ws=None), dict(ws=P256 + 128), dict(size=n.value - 1)):
        assert back(**kw) == INVALID


def test_linear_ce_of_no_rows_is_no_error(lib):
    assert lib.elasto_op_linear_ce(ce(rows=0, x=None, labels=None), None, None, None, 0, None) == 0


def test_linear_ce_workspace_is_bounded(lib):
    """The logits' gradient of one piece and the sums of dx, not a matrix of rows x classes."""
    n = ctypes.c_int64()
    assert lib.elasto_linear_ce_workspace(ce(rows=16384, classes=1 << 20, dim=4096, ldx=4096, ldw=4096), 1,
                                          ctypes.byref(n)) == 0
    assert n.value < (1 << 30)


def test_linear_ce_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 16), torch.zeros(10, 16)
    for bad_x, bad_w in ((x[0], w), (x, torch.zeros(10, 8)), (x, w.to(torch.bfloat16)),
                         (x.t(), w), (x.half(), w.half())):
        with pytest.raises(ValueError):
            ffi.linear_cross_entropy_workspace(bad_x, bad_w)
