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


# ------------------------------------------------------------------------ clipping

def grads(*entries):
    return (ffi.Grad * max(1, len(entries)))(*[ffi.Grad(*e) for e in entries])


def clip(lib, g, o=None, n=None, max_norm=1.0, stats=P256, ws=P256, size=1 << 40):
    o = g if o is None else o
    return lib.elasto_op_clip_gradients(g, o, len(g) if n is None else n, max_norm, stats, ws, size, None)


GOOD = (P256, 1000, 0), (2 * P256, 77, 1)


@pytest.mark.parametrize("bad", [(None, 5, 0), (P256 + 2, 5, 0), (P256 + 1, 5, 1), (P256, -1, 0),
                                 (P256, 5, 2), (P256, 1 << 40, 0)])
def test_clip_refuses_bad_tensors(lib, bad):
    n = ctypes.c_int64()
    g = grads(GOOD[0], bad)
    assert lib.elasto_grad_norm_workspace(g, 2, ctypes.byref(n)) == INVALID
    assert lib.elasto_op_grad_norm(g, 2, P256, P256, 1 << 40, None) == INVALID
    assert clip(lib, g) == INVALID
    assert clip(lib, grads(*GOOD), g) == INVALID


def test_clip_refuses_bad_arguments(lib):
    n = ctypes.c_int64()
    g = grads(*GOOD)
    assert lib.elasto_grad_norm_workspace(g, 2, None) == INVALID
    assert lib.elasto_grad_norm_workspace(g, -1, ctypes.byref(n)) == INVALID
    assert lib.elasto_grad_norm_workspace(None, 1, ctypes.byref(n)) == INVALID
    assert lib.elasto_grad_norm_workspace(g, (1 << 20) + 1, ctypes.byref(n)) == INVALID
    assert lib.elasto_grad_norm_workspace(g, 2, ctypes.byref(n)) == 0 and n.value > 0
    for norm, ws, size in ((None, P256, n.value), (P256 + 2, P256, n.value), (P256, None, n.value),
                           (P256, P256 + 8, n.value), (P256, P256, n.value - 1)):
        assert lib.elasto_op_grad_norm(g, 2, norm, ws, size, None) == INVALID
    for kw in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(stats=None),
               dict(stats=P256 + 2), dict(ws=None), dict(size=n.value - 1)):
        assert clip(lib, g, **kw) == INVALID


@pytest.mark.parametrize("out", [
    (GOOD[0], (2 * P256, 76, 1)), (GOOD[0], (2 * P256, 77, 0)),          # other sizes, other types
    ((P256 + 4, 1000, 0), GOOD[1]),                                      # over its own gradient, shifted
    ((2 * P256 + 64, 1000, 0), GOOD[1]),                                 # over the other result
    ((4 * P256, 1000, 0), (P256 + 400, 77, 1)),                          # over the other gradient
    ((4 * P256, 1000, 0), (4 * P256 + 3998, 77, 1))])
def test_clip_refuses_results_that_overlap(lib, out):
    assert clip(lib, grads(*GOOD), grads(*out)) == INVALID


def test_clip_refuses_the_same_tensor_twice(lib):
    assert clip(lib, grads(GOOD[0], GOOD[0])) == INVALID


def test_grad_lists_refuse_what_is_not_one_run():
    torch = pytest.importorskip("torch")
    t = torch.zeros(6, 8)
    for bad in (t[:, :4], t[::2], t.half(), torch.zeros(1).expand(5)):
        with pytest.raises(ValueError):
            ffi.GradList([bad])
    assert len(ffi.GradList([t.t(), t[2:4], torch.zeros(3, 0), torch.zeros(())])) == 4


def test_grad_lists_follow_types_and_strides_at_the_same_place():
    """Another type, order or extent at the address and of the size that the list has seen."""
    torch = pytest.importorskip("torch")
    buf = torch.zeros(128)
    t, other = buf[:60].view(6, 10), torch.zeros(5)
    g = ffi.GradList([other, t])

    def entry():
        e = g.entries()[1]
        return e.data, e.count, e.dtype

    place = buf.data_ptr()
    assert entry() == (place, 60, ffi.FP32) and g.changes == 1
    g.entries()
    assert g.changes == 1
    g.paired = "a list"
    t.t_()                                             # the elements in another order
    assert entry() == (place, 60, ffi.FP32) and g.changes == 2 and g.paired is None
    t.data = buf[:60].view(10, 6)                      # (that order's shape, another order)
    g.entries()
    assert g.changes == 3
    t.data = buf.view(torch.bfloat16)[:60].view(10, 6)   # half of the bytes
    assert entry() == (place, 60, ffi.BF16) and g.changes == 4
    for bad in (buf.as_strided((10, 6), (7, 1)),       # beyond its elements
                buf.as_strided((12, 5), (6, 1)),       # (strides as they were)
                buf[:1].expand(60), buf.view(torch.int32)[:60].view(10, 6),
                buf.view(torch.float16)[:60].view(10, 6)):
        before = t.data
        t.data = bad
        for _ in range(2):
            with pytest.raises(ValueError):
                g.entries()
        t.data = before
        assert entry() == (place, 60, ffi.BF16)
    # A list that was refused half way is laid out again when its tensors are back.
    was = other.data
    other.data, t.data = torch.zeros(9), buf.as_strided((10, 6), (7, 1))
    with pytest.raises(ValueError):
        g.entries()
    other.data, t.data = was, before
    assert (g.entries()[0].data, g.entries()[0].count) == (was.data_ptr(), 5)
    assert entry() == (place, 60, ffi.BF16)


# --------------------------------------------------- queries and keys on several axes

def heads(data=P256, b=1 << 16, t=768, h=64):
    return ffi.Heads(data, b, t, h)


def axes_desc(axes=3, in_turn=0, norm=1, sections=(12, 10, 10, 0), **kw):
    d = dict(dtype=1, batch=2, tokens=8, q_heads=12, kv_heads=4, head_dim=64, rot_dim=64, interleaved=0,
             table_rows=8, eps=1e-6, positions=P256, lens=None, cos=P256, sin=P256, q_gamma=P256, k_gamma=P256)
    d.update(kw)
    base = ffi.QkNorm(*[d[n] for n, _ in ffi.QkNorm._fields_])
    return ffi.QkAxes(base, axes, in_turn, norm, (ctypes.c_int32 * 4)(*sections))


NO_GAMMA = dict(q_gamma=None, k_gamma=None)


@pytest.mark.parametrize("kw", [
    dict(axes=0), dict(axes=5), dict(axes=-1), dict(axes=2), dict(sections=(12, 10, 9, 1)),
    dict(sections=(42, -10, 0, 0)), dict(sections=(1 << 30, 1 << 30, 1 << 30, 0)), dict(positions=None),
    dict(positions=P256 + 2), dict(norm=0), dict(cos=None), dict(sin=P256 + 1), dict(table_rows=0), dict(eps=0.0),
    dict(head_dim=72), dict(rot_dim=8, sections=(4, 0, 0, 0)), dict(dtype=5), dict(tokens=-1)])
def test_axes_refuses_bad_descriptions(lib, kw):
    h = heads()
    assert lib.elasto_op_qk_norm_rotate_axes(axes_desc(**kw), h, h, h, h, None) == INVALID
    assert lib.elasto_op_qk_norm_rotate_axes_bwd(axes_desc(**kw), h, h, h, h, h, h, None, None, None, 0,
                                                 None) == INVALID
    assert lib.elasto_last_error()


def test_axes_refuses_bad_tensors(lib):
    h = heads()
    for i in range(4):
        for bad in (None, heads(None), heads(P256 + 8), heads(b=4), heads(t=772)):
            args = [h] * 4
            args[i] = bad
            assert lib.elasto_op_qk_norm_rotate_axes(axes_desc(), *args, None) == INVALID
    for norm in (0, 1):
        d = axes_desc(norm=norm, **({} if norm else NO_GAMMA))
        for i in range(6):
            if not norm and i < 2:       # q and k are not used
                continue
            args = [h] * 6
            args[i] = None
            assert lib.elasto_op_qk_norm_rotate_axes_bwd(d, *args, None, None, None, 0, None) == INVALID
    assert lib.elasto_op_qk_norm_rotate_axes(None, h, h, h, h, None) == INVALID
    # Gradients of weights that are not there, and a workspace that is too short for those that are.
    assert lib.elasto_op_qk_norm_rotate_axes_bwd(axes_desc(norm=0, **NO_GAMMA), h, h, h, h, h, h, P256, None, P256,
                                                 1 << 30, None) == INVALID
    assert lib.elasto_op_qk_norm_rotate_axes_bwd(axes_desc(), h, h, h, h, h, h, P256, None, P256, 16, None) == INVALID


def test_axes_of_no_tokens_is_no_error(lib):
    for kw in (dict(batch=0), dict(tokens=0)):
        d = axes_desc(**kw, positions=None, cos=None, sin=None)
        assert lib.elasto_op_qk_norm_rotate_axes(d, None, None, None, None, None) == 0


# ------------------------------------------------------------------- between blocks

def rows(data=P256, b=1 << 16, t=768):
    return ffi.Rows(data, b, t)


def block(**kw):
    d = dict(dtype=1, stream_dtype=0, kind=1, batch=2, tokens=8, dim=64, post_norm=1, gate_per_sequence=0,
             residual_scale=1.0, eps=1e-6, pre_gamma=P256, pre_beta=P256, post_gamma=P256, post_beta=P256,
             gate=P256, lens=None)
    d.update(kw)
    return ffi.BlockNorm(*[d[n] for n, _ in ffi.BlockNorm._fields_])


def block_fwd(lib, d, x=rows(), y=rows(), x_out=rows(), u=rows()):
    return lib.elasto_op_block_norm(d, x, y, x_out, u, None)


def block_bwd(lib, d, x_out=rows(), y=rows(), dx_out=rows(), du=rows(), dx=rows(), dy=rows(), grads=(P256,) * 5,
              ws=P256, size=1 << 40):
    return lib.elasto_op_block_norm_bwd(d, x_out, y, dx_out, du, dx, dy, *grads, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(stream_dtype=3), dict(dtype=0, stream_dtype=1), dict(kind=2), dict(kind=-1), dict(batch=-1),
    dict(tokens=-1), dict(dim=0), dict(dim=16385), dict(batch=1 << 13, tokens=1 << 13), dict(eps=0.0),
    dict(eps=1e-39), dict(eps=math.inf), dict(eps=math.nan), dict(residual_scale=math.inf),
    dict(residual_scale=math.nan), dict(post_norm=0), dict(kind=0), dict(pre_gamma=P256 + 2),
    dict(post_beta=P256 + 1), dict(gate=P256 + 2), dict(lens=P256 + 2)])
def test_block_norm_refuses_bad_descriptions(lib, kw):
    assert block_fwd(lib, block(**kw)) == INVALID
    assert block_bwd(lib, block(**kw)) == INVALID
    assert lib.elasto_last_error()


def test_block_norm_refuses_bad_tensors(lib):
    for bad in (rows(P256 + 1), rows(b=-768), rows(t=-64)):
        for name in ("x", "y", "x_out", "u"):
            assert block_fwd(lib, block(), **{name: bad}) == INVALID
        for name in ("x_out", "y", "dx_out", "du", "dx", "dy"):
            assert block_bwd(lib, block(), **{name: bad}) == INVALID
    for bad in (rows(b=63), rows(t=0), rows(t=63)):      # rows that overlap
        for name in ("x_out", "u"):
            assert block_fwd(lib, block(), **{name: bad}) == INVALID
        for name in ("dx", "dy"):
            assert block_bwd(lib, block(), **{name: bad}) == INVALID
    assert block_fwd(lib, None) == INVALID and block_bwd(lib, None) == INVALID
    assert block_fwd(lib, block(), x=None) == INVALID
    assert block_fwd(lib, block(), x_out=None, u=None) == INVALID
    assert block_fwd(lib, block(), y=None) == INVALID                       # a norm and a gate of nothing
    assert block_fwd(lib, block(post_norm=0, post_gamma=None, post_beta=None), y=None) == INVALID


def test_block_norm_backward_refuses_what_does_not_go_together(lib):
    none = (None,) * 5
    assert block_bwd(lib, block(), x_out=None) == INVALID                   # du needs it
    assert block_bwd(lib, block(), dx_out=None, du=None, grads=none) == INVALID
    assert block_bwd(lib, block(), y=None, dy=None, grads=none) == INVALID
    assert block_bwd(lib, block(), du=None) == INVALID                      # gradients of pre_gamma and pre_beta
    bare = dict(post_norm=0, post_gamma=None, post_beta=None)
    assert block_bwd(lib, block(**bare)) == INVALID                         # of weights that are not there
    assert block_bwd(lib, block(gate=None), grads=(None,) * 4 + (P256,)) == INVALID
    assert block_bwd(lib, block(kind=0, pre_beta=None, post_beta=None), grads=(None, P256, None, None, None)) == INVALID
    assert block_bwd(lib, block(**bare, gate=None), y=None, grads=none) == INVALID     # dy of no y
    for i in range(5):
        grads = [None] * 5
        grads[i] = P256 + 2
        assert block_bwd(lib, block(), grads=grads) == INVALID
    n = ctypes.c_int64()
    assert lib.elasto_block_norm_workspace(block(), ctypes.byref(n)) == 0 and n.value > 0
    assert lib.elasto_block_norm_workspace(block(), None) == INVALID
    assert lib.elasto_block_norm_workspace(block(dim=0), ctypes.byref(n)) == INVALID
    for ws, size in ((None, n.value), (P256 + 8, n.value), (P256, n.value - 1)):
        assert block_bwd(lib, block(), ws=ws, size=size) == INVALID


def test_block_norm_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 3, 8)
    for args in ((x[0], None), (x, torch.zeros(3, 8)), (x, torch.zeros(7))):
        with pytest.raises(ValueError):
            ffi.block_norm_workspace(*args)


def test_block_norm_of_no_tokens_is_no_error(lib):
    for kw in (dict(batch=0), dict(tokens=0)):
        assert block_fwd(lib, block(**kw), None, None, None, None) == 0
        assert block_bwd(lib, block(**kw), None, None, None, None, None, None, (None,) * 5, None, 0) == 0
