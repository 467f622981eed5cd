"""The operators on token sequences refuse bad calls before any pointer is
used or any HIP call is made: checked through the C ABI with addresses that
nothing may touch, and through the Python binding with CPU tensors' shapes."""
import ctypes
import math
import os

import pytest

from paper_2609_10018_amd import ffi

P16 = 1 << 20
INVALID = 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ffi.LIB_PATH):
        pytest.skip("library not built")
    return ffi.load_library()


def heads(data=P16, b=1 << 16, t=768, h=64):
    return ffi.Heads(data, b, t, h)


# ------------------------------------------------------------- queries and keys

def qk_desc(**kw):
    d = dict(dtype=1, batch=2, tokens=8, q_heads=12, kv_heads=4, head_dim=64, rot_dim=64,
             interleaved=0, table_rows=8, eps=1e-6, positions=None, lens=None, cos=P16, sin=P16,
             q_gamma=P16, k_gamma=P16)
    d.update(kw)
    return ffi.QkNorm(*[d[n] for n, _ in ffi.QkNorm._fields_])


def qk(lib, q=heads(), k=heads(), q_out=heads(), k_out=heads(), **kw):
    return lib.elasto_op_qk_norm_rotate(qk_desc(**kw), q, k, q_out, k_out, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(batch=-1), dict(tokens=-1), dict(q_heads=0, kv_heads=0), dict(q_heads=-1),
    dict(head_dim=72), dict(head_dim=8), dict(head_dim=272), dict(rot_dim=8), dict(rot_dim=80),
    dict(rot_dim=-16), dict(eps=0.0), dict(eps=1e-39), dict(eps=math.nan), dict(eps=math.inf), dict(cos=None),
    dict(sin=None), dict(table_rows=0), dict(table_rows=7), dict(cos=P16 + 2),
    dict(positions=P16 + 2), dict(lens=P16 + 1), dict(q_gamma=P16 + 2),
    dict(batch=1 << 20, tokens=1 << 20)])
def test_qk_norm_refuses_bad_descriptions(lib, kw):
    assert qk(lib, **kw) == INVALID
    assert lib.elasto_last_error()


@pytest.mark.parametrize("side", ["q", "k", "q_out", "k_out"])
@pytest.mark.parametrize("bad", [None, heads(None), heads(P16 + 8), heads(b=4), heads(t=772),
                                 heads(h=60)])
def test_qk_norm_refuses_bad_tensors(lib, side, bad):
    assert qk(lib, **{side: bad}) == INVALID


@pytest.mark.parametrize("side", ["q_out", "k_out"])
@pytest.mark.parametrize("bad", [heads(b=0), heads(t=0), heads(h=0), heads(h=48), heads(t=-768)])
def test_qk_norm_refuses_overlapping_results(lib, side, bad):
    assert qk(lib, **{side: bad}) == INVALID


def test_qk_norm_backward_refuses_a_short_workspace(lib):
    n = ctypes.c_int64()
    assert lib.elasto_qk_norm_rotate_workspace(qk_desc(), ctypes.byref(n)) == 0 and n.value > 0
    assert lib.elasto_qk_norm_rotate_workspace(qk_desc(), None) == INVALID
    assert lib.elasto_qk_norm_rotate_workspace(None, ctypes.byref(n)) == INVALID
    h = heads()
    for ws, size in ((None, 1 << 20), (P16, 0), (P16 + 4, 1 << 30)):
        assert lib.elasto_op_qk_norm_rotate_bwd(qk_desc(), h, h, h, h, h, h, P16, P16, ws, size,
                                                None) == INVALID
    assert lib.elasto_op_qk_norm_rotate_bwd(qk_desc(), h, h, None, h, h, h, None, None, None, 0,
                                            None) == INVALID


def test_nothing_to_do_is_no_error(lib):
    none = [None] * 4
    assert lib.elasto_op_qk_norm_rotate(qk_desc(batch=0), *none, None) == 0
    assert lib.elasto_op_qk_norm_rotate(qk_desc(tokens=0), *none, None) == 0
    assert lib.elasto_op_window_attention(win_desc(batch=0), *none, None, None, 0, None) == 0
    assert lib.elasto_op_window_attention(win_desc(q_tokens=0), *none, None, None, 0, None) == 0
    assert lib.elasto_op_window_attention_bwd(win_desc(q_tokens=0, k_tokens=0), *none, None, *none,
                                              None, 0, None) == 0
    assert lib.elasto_op_top_logits(1, None, 10, 0, 10, 2, None, None, None) == 0
    assert lib.elasto_op_distill(1, None, 10, 0, 10, None, None, 2, None, None, 1.0, 1.0, 1.0, None,
                                 1, None, 10, None) == 0


# ------------------------------------------------------------------- attention

def win_desc(**kw):
    d = dict(dtype=1, batch=2, q_tokens=300, k_tokens=300, heads=12, kv_heads=4, head_dim=64,
             causal=1, window=100, sinks=4, scale=0.125, q_lens=None, k_lens=None)
    d.update(kw)
    return ffi.Window(*[d[n] for n, _ in ffi.Window._fields_])


BIG = 1 << 34


def attn(lib, q=heads(), k=heads(), v=heads(), o=heads(), lse=P16, ws=P16, size=BIG, **kw):
    return lib.elasto_op_window_attention(win_desc(**kw), q, k, v, o, lse, ws, size, None)


def attn_bwd(lib, lse=P16, ws=P16, size=BIG, desc=None, **kw):
    t = {n: heads() for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")}
    t.update(kw)
    return lib.elasto_op_window_attention_bwd(desc or win_desc(), t["q"], t["k"], t["v"], t["o"], lse,
                                              t["dout"], t["dq"], t["dk"], t["dv"], ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=7), dict(head_dim=32), dict(head_dim=96), dict(batch=-1), dict(q_tokens=-1),
    dict(k_tokens=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=5), dict(window=0),
    dict(window=-3), dict(sinks=-1), dict(sinks=65), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-31), dict(scale=1e31),
    dict(q_lens=P16 + 2), dict(k_lens=P16 + 1),
    dict(k_tokens=(1 << 29) + 1), dict(q_tokens=1 << 29), dict(batch=1 << 28), dict(lse=P16 + 2)])
def test_window_attention_refuses_bad_descriptions(lib, kw):
    assert attn(lib, **kw) == INVALID
    lse = kw.pop("lse", P16)
    assert attn_bwd(lib, desc=win_desc(**kw), lse=lse) == INVALID


@pytest.mark.parametrize("side", ["q", "k", "v", "o"])
@pytest.mark.parametrize("bad", [None, heads(None), heads(P16 + 8), heads(b=4), heads(t=772),
                                 heads(h=60)])
def test_window_attention_refuses_bad_tensors(lib, side, bad):
    assert attn(lib, **{side: bad}) == INVALID
    assert attn_bwd(lib, **{side: bad}) == INVALID


@pytest.mark.parametrize("side", ["dout", "dq", "dk", "dv"])
def test_window_attention_backward_refuses_bad_gradients(lib, side):
    assert attn_bwd(lib, **{side: None}) == INVALID
    assert attn_bwd(lib, **{side: heads(P16 + 4)}) == INVALID
    if side != "dout":
        for bad in (heads(b=0), heads(t=0), heads(h=0), heads(h=56)):
            assert attn_bwd(lib, **{side: bad}) == INVALID
    assert attn_bwd(lib, lse=None) == INVALID


def test_window_attention_refuses_tiles_wider_than_four_gigabytes(lib):
    far = heads(t=1 << 25)                           # bf16: 64 tokens are 4 GiB apart
    for side in "kv":
        assert attn(lib, **{side: far}) == INVALID
        assert attn_bwd(lib, **{side: far}) == INVALID
    for side in ("q", "dout"):
        assert attn_bwd(lib, **{side: far}) == INVALID
        assert attn_bwd(lib, **{side: heads(h=1 << 30)}) == INVALID


def test_heads_read_one_at_a_time_may_lie_any_distance_apart(lib):
    """Only the heads of a group are reached at 32-bit offsets from one another.  The calls end at
    the workspace, which is looked at behind the tensors."""
    far = heads(t=64, h=1 << 31)                     # bf16: 4 GiB from head to head
    for side in "kv":
        assert attn(lib, ws=None, q_tokens=1, k_tokens=8192, window=4096, **{side: far}) == INVALID
        assert b"the workspace holds" in lib.elasto_last_error()
        assert attn_bwd(lib, ws=None, **{side: far}) == INVALID
        assert b"the workspace holds" in lib.elasto_last_error()
    for side in ("q", "dout"):
        assert attn_bwd(lib, ws=None, desc=win_desc(heads=4), **{side: far}) == INVALID
        assert b"the workspace holds" in lib.elasto_last_error()
        assert attn_bwd(lib, ws=None, **{side: far}) == INVALID
        assert b"4 GiB" in lib.elasto_last_error()


def test_more_work_than_a_launch_holds_is_refused(lib):
    many = dict(batch=1 << 20, heads=16, kv_heads=16, q_tokens=1, k_tokens=10)
    assert attn(lib, **many) == INVALID
    many["q_tokens"] = 1 << 12
    assert attn_bwd(lib, desc=win_desc(**many), size=1 << 60) == INVALID
    many.update(q_tokens=1, k_tokens=1 << 12)
    assert attn_bwd(lib, desc=win_desc(**many), size=1 << 60) == INVALID
    assert qk(lib, batch=1 << 13, tokens=(1 << 12) + 1) == INVALID


def test_negative_strides_are_refused(lib):
    for bad in (heads(b=-64), heads(t=-64), heads(h=-64)):
        assert attn(lib, q=bad) == INVALID
        assert qk(lib, k=bad) == INVALID


def test_window_attention_refuses_a_short_workspace(lib):
    n = ctypes.c_int64()
    one = dict(q_tokens=1, k_tokens=8192, window=4096)
    assert lib.elasto_window_attention_workspace(win_desc(**one), 0, ctypes.byref(n)) == 0
    assert n.value > 0
    assert attn(lib, size=n.value - 1, **one) == INVALID
    assert attn(lib, ws=None, **one) == INVALID
    assert attn(lib, ws=P16 + 16, **one) == INVALID
    assert lib.elasto_window_attention_workspace(win_desc(), 1, ctypes.byref(n)) == 0 and n.value > 0
    assert attn_bwd(lib, size=n.value - 1) == INVALID
    assert attn_bwd(lib, ws=None) == INVALID
    assert lib.elasto_window_attention_workspace(win_desc(), 0, None) == INVALID
    assert lib.elasto_window_attention_workspace(win_desc(window=0), 0, ctypes.byref(n)) == INVALID


# ---------------------------------------------------------------------- logits

@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(rows=-1), dict(classes=0), dict(ld=999), dict(top=0), dict(top=257),
    dict(classes=10, top=11), dict(logits=None), dict(values=None), dict(indices=None),
    dict(logits=P16 + 1), dict(values=P16 + 2), dict(indices=P16 + 2)])
def test_top_logits_refuses_bad_calls(lib, kw):
    a = dict(dtype=1, logits=P16, ld=1000, rows=4, classes=1000, top=16, values=P16, indices=P16)
    a.update(kw)
    assert lib.elasto_op_top_logits(*a.values(), None) == INVALID


DISTILL = dict(dtype=1, logits=P16, ld=1000, rows=4, classes=1000, values=P16, indices=P16, top=16,
               labels=P16, weight=P16, temperature=2.0, alpha=0.5, scale=1.0, loss=P16,
               grad_dtype=1, dlogits=P16 + 4096, ldg=1000)


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(grad_dtype=-1), dict(rows=-1), dict(classes=0), dict(ld=999), dict(ldg=999),
    dict(top=-1), dict(top=257), dict(top=0), dict(temperature=0.0), dict(temperature=-1.0),
    dict(temperature=math.inf), dict(temperature=math.nan), dict(alpha=-0.1), dict(alpha=1.1),
    dict(alpha=math.nan), dict(scale=math.inf), dict(scale=math.nan), dict(labels=None),
    dict(logits=None), dict(loss=None), dict(values=None), dict(indices=None),
    dict(logits=P16 + 1), dict(dlogits=P16 + 1), dict(loss=P16 + 2), dict(values=P16 + 2),
    dict(indices=P16 + 2), dict(labels=P16 + 2), dict(weight=P16 + 2),
    dict(dlogits=P16, grad_dtype=0), dict(dlogits=P16, ldg=1008)])
def test_distill_refuses_bad_calls(lib, kw):
    a = dict(DISTILL)
    a.update(kw)
    assert lib.elasto_op_distill(*a.values(), None) == INVALID


def test_growth_step_distill_refuses_a_missing_context(lib):
    assert lib.elasto_growth_step_distill(None, 0, P16, P16, P16, P16, 8, 1.0, 0.5, 1, 0.1, 1.0,
                                          None, None) == INVALID


# ------------------------------------------------------------------- the binding

def test_binding_refuses_shapes_types_and_devices(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    q = torch.zeros(2, 5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        ffi.op_qk_norm_rotate(q, q, q, q)                        # not on the GPU
    monkeypatch.setattr(ffi, "_same_device", lambda *t: None)
    bad = [
        lambda: ffi.op_qk_norm_rotate(q, q, q[:, :4], q),
        lambda: ffi.op_qk_norm_rotate(q, q, q.float(), q),
        lambda: ffi.op_qk_norm_rotate(q.half(), None, q.half(), None),
        lambda: ffi.op_qk_norm_rotate(q, q, q.transpose(2, 3), q),
        lambda: ffi.op_qk_norm_rotate(q, q, q, q, cos=torch.zeros(9, 32)),
        lambda: ffi.op_qk_norm_rotate(q, q, q, q, q_gamma=torch.zeros(63)),
        lambda: ffi.op_qk_norm_rotate(q, q, q, q, q_gamma=torch.zeros(64).double()),
        lambda: ffi.op_qk_norm_rotate(q, q, q, q, positions=torch.zeros(2, 4, dtype=torch.int32)),
        lambda: ffi.op_qk_norm_rotate(q, q, q, q, lens=torch.zeros(2, dtype=torch.int64)),
        lambda: ffi.op_qk_norm_rotate_bwd(q, q, q, q, q, q, torch.zeros(60)),
        lambda: ffi.op_window_attention(q, q, q, q[:, :, :2], 8),
        lambda: ffi.op_window_attention(q, q[:1], q, q, 8),
        lambda: ffi.op_window_attention(q, q, q.float(), q, 8),
        lambda: ffi.op_window_attention(q, q, q, q, 8, lse=torch.zeros(2, 4, 4)),
        lambda: ffi.op_window_attention(q, q, q, q, 8, q_lens=torch.zeros(3, dtype=torch.int32)),
        lambda: ffi.op_window_attention_bwd(q, q, q, q, torch.zeros(2, 4, 5), q, q, q[:, :3], q, 8),
        lambda: ffi.op_top_logits(torch.zeros(4, 10).T, torch.zeros(10, 2), torch.zeros(10, 2)),
        lambda: ffi.op_top_logits(torch.zeros(4, 10), torch.zeros(3, 2),
                                  torch.zeros(3, 2, dtype=torch.int32)),
        lambda: ffi.op_distill(torch.zeros(4, 10), torch.zeros(4, 2),
                               torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4)),
        lambda: ffi.op_distill(torch.zeros(4, 10), torch.zeros(4, 2),
                               torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4)),
        lambda: ffi.op_distill(torch.zeros(4, 10), torch.zeros(4, 2),
                               torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4),
                               dlogits=torch.zeros(4, 9)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was accepted")


def test_binding_refuses_sizes_beyond_32_bits(lib, monkeypatch):
    """ctypes cuts integers off at 32 bits: 2^32 + 8 keys would be 8.  (Tensors without that much
    memory: expanded, or of shapes alone.)"""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(ffi, "_same_device", lambda *t: None)
    n = 2 ** 32 + 8
    q = torch.zeros(1, 8, 2, 64)

    def wide(axis, size=n):
        shape = [1, 1, 1, 64]
        shape[axis] = size
        return torch.zeros(1, 1, 1, 64).expand(shape)

    def meta(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    i32 = torch.int32
    for call in (
            lambda: ffi.window_attention_workspace(q, wide(1), 8),
            lambda: ffi.window_attention_workspace(wide(1), q[:, :, :1], 8),
            lambda: ffi.window_attention_workspace(wide(0), wide(0), 8),
            lambda: ffi.window_attention_workspace(wide(2), wide(2, 1), 8),
            lambda: ffi.qk_norm_rotate_workspace(wide(0), None),
            lambda: ffi.qk_norm_rotate_workspace(None, wide(1)),
            lambda: ffi.qk_norm_rotate_workspace(wide(1, 3), wide(2)),
            lambda: ffi.op_qk_norm_rotate(q, None, q, None, cos=meta(n, 32), sin=meta(n, 32)),
            lambda: ffi.op_top_logits(meta(1, n), meta(1, 2), meta(1, 2, dtype=i32)),
            lambda: ffi.op_top_logits(meta(1, 9), meta(1, n), meta(1, n, dtype=i32)),
            lambda: ffi.op_distill(meta(1, n), meta(1, 2), meta(1, 2, dtype=i32), meta(1)),
            lambda: ffi.op_distill(meta(1, 9), meta(1, n), meta(1, n, dtype=i32), meta(1))):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    for kw in (dict(window=8, sinks=n), dict(window=8, sinks=8 - 2 ** 32), dict(window=8 - 2 ** 32)):
        with pytest.raises(ffi.ElastoError):
            ffi.window_attention_workspace(q, q, **kw)
    assert ffi.window_attention_workspace(q, q, n) == ffi.window_attention_workspace(q, q, 8)


def test_binding_asks_torch_for_the_current_device_at_each_call(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(ffi, "_torch", None)
    for device in (3, 5):
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "current_device", lambda d=device: d)
            assert ffi._same_device() == device
