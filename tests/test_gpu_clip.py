"""The global norm of many tensors and their clipping, against 64 bits.

Tolerances.  Squares are exact in 64 bits (24 or 8 bits each) and summed there: with n
elements the sum is off by at most n 2^-53 relative, below 2^-25 for n < 2^28, and its root
is rounded to fp32 once: the norm is off by at most 2^-23 relative.  The factor: two more
roundings in 64 bits and one to fp32.  A result is the gradient times that factor in fp32,
rounded to its type: finfo(type).eps / 2 + 3 * 2^-24 relative (and half of the type's smallest step).
"""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


def tensors(sizes, seed=0, offset=0, scale=1e-2):
    """[(size, dtype)] as views at odd places of larger buffers, whose rest holds NaN."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, (n, dt) in enumerate(sizes):
        at = (offset * (i + 1)) % 11
        buf = torch.full((n + 32,), math.nan, dtype=dt, device="cuda")
        buf[at:at + n] = (torch.randn(n, generator=g) * scale).to(dt).cuda()
        out.append(buf[at:at + n])
    return out


def norm_of(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def space(ts):
    return torch.full((ffi.grad_norm_workspace(ts),), 0xff, dtype=torch.uint8, device="cuda")


def check(got, ts, max_norm, stats):
    ref = norm_of(ts)
    norm, factor = stats.tolist()
    assert abs(norm - ref) <= 2.0 ** -23 * ref
    want = min(1.0, max_norm / ref) if ref else 1.0
    assert abs(factor - want) <= 2.0 ** -23 * want
    for t, o in zip(ts, got):
        w = t.double() * want
        tol = (torch.finfo(t.dtype).eps / 2 + 3 * 2.0 ** -24) * w.abs() + torch.finfo(t.dtype).tiny
        assert ((o.double() - w).abs() <= tol).all()


LISTS = [
    [(1, F32)], [(1, BF)], [(7, BF), (9, F32), (16, BF)], [(8192, BF)], [(8193, BF), (4097, F32)],
    [(100000, F32), (3, BF), (0, F32), (70001, BF), (1, F32)],
    [(1 + 37 * i % 900, (BF, F32)[i % 2]) for i in range(500)],
    [(5_000_011, BF), (3_000_003, F32)],
]


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("sizes", LISTS, ids=range(len(LISTS)))
def test_norm_and_clipping(sizes, offset):
    ts = tensors(sizes, offset=offset)
    ref = norm_of(ts)
    norm, stats = torch.empty(1, device="cuda"), torch.empty(2, device="cuda")
    ffi.op_grad_norm(ts, norm, workspace=space(ts))
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref
    for share in (0.3, 1.5):
        # Results at places of their own, at other alignments too.
        out = tensors(sizes, seed=1, offset=offset + (share > 1))
        around = [o._base.clone() for o in out]
        ffi.op_clip_gradients(ts, share * ref, stats, out=out, workspace=space(ts))
        check(out, ts, share * ref, stats)
        for o, before in zip(out, around):
            now = o._base.clone()
            at = o.storage_offset()
            now[at:at + o.numel()] = 0
            before[at:at + o.numel()] = 0
            assert torch.equal(now.isnan(), before.isnan()) and not now.nan_to_num(0.0).any()
    before = [t.clone() for t in ts]
    ffi.op_clip_gradients(ts, 0.3 * ref, stats, workspace=space(ts))
    check(ts, before, 0.3 * ref, stats)


def test_nothing_to_clip_leaves_the_bits():
    ts = tensors(LISTS[5])
    before = [t.clone() for t in ts]
    stats = torch.empty(2, device="cuda")
    for limit in (2 * norm_of(ts), math.inf):
        ffi.op_clip_gradients(ts, limit, stats, workspace=space(ts))
        assert float(stats[1]) == 1.0 and all(torch.equal(a, b) for a, b in zip(ts, before))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_no_number_scales_nothing(bad):
    ts = tensors(LISTS[5])
    ts[0][77] = bad
    before = [t.clone() for t in ts]
    out = tensors(LISTS[5], seed=4)
    stats = torch.empty(2, device="cuda")
    ffi.op_clip_gradients(ts, 0.1, stats, workspace=space(ts))
    assert not math.isfinite(float(stats[0])) and float(stats[1]) == 0.0
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(ts, before))
    ffi.op_clip_gradients(ts, 0.1, stats, out=out, workspace=space(ts))
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(out, before))


@pytest.mark.parametrize("size", [1e30, 1e-30])
def test_squares_beyond_32_bits(size):
    ts = tensors([(1000, F32), (500, BF)], scale=size)
    norm = torch.empty(1, device="cuda")
    ffi.op_grad_norm(ts, norm, workspace=space(ts))
    assert abs(float(norm) - norm_of(ts)) <= 2.0 ** -23 * norm_of(ts)


def test_zeros_and_empty_lists():
    stats, norm = torch.full((2,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    for ts in ([], [torch.empty(0, device="cuda")], [torch.zeros(100, device="cuda", dtype=BF)]):
        ffi.op_grad_norm(ts, norm, workspace=space(ts))
        ffi.op_clip_gradients(ts, 1.0, stats, workspace=space(ts))
        assert float(norm) == 0.0 and stats.tolist() == [0.0, 1.0]


def test_a_list_is_used_again_and_follows_its_tensors():
    ts = tensors([(4000, F32), (513, BF)])
    g = ffi.GradList(ts)
    ws, stats = space(g), torch.empty(2, device="cuda")
    ref = norm_of(ts)
    ffi.op_clip_gradients(g, 0.5 * ref, stats, workspace=ws)
    ffi.op_clip_gradients(g, 0.5 * ref, stats, workspace=ws)
    # (0.5 of the norm, each element rounded by half a step of its type)
    assert abs(float(stats[0]) - 0.5 * ref) <= 2.0 ** -8 * ref
    ts[0].data = torch.ones(4000, device="cuda")
    ffi.op_grad_norm(g, stats[:1], workspace=ws)
    assert abs(float(stats[0]) - norm_of(ts)) <= 2.0 ** -23 * norm_of(ts)


def test_dense_tensors_of_any_order():
    t = torch.randn(6, 5, 4, device="cuda").permute(2, 0, 1)
    stats = torch.empty(2, device="cuda")
    before = t.clone()
    ffi.op_clip_gradients([t], 0.25 * norm_of([before]), stats, workspace=space([t]))
    check([t], [before], 0.25 * norm_of([before]), stats)


def test_captured_and_replayed():
    ts = tensors(LISTS[6])
    out = tensors(LISTS[6], seed=9)
    stats, ws = torch.empty(2, device="cuda"), space(ts)
    g, o = ffi.GradList(ts), ffi.GradList(out)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ffi.op_clip_gradients(g, 0.1, stats, out=o, workspace=ws)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ffi.op_clip_gradients(g, 0.1, stats, out=o, workspace=ws)
    for i in range(4):
        for t in ts:
            t.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        got, st = [t.clone() for t in out], stats.clone()
        ffi.op_clip_gradients(g, 0.1, stats, out=o, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(st, stats) and all(torch.equal(a, b) for a, b in zip(got, out))
        check(out, ts, 0.1, stats)


def test_lists_that_have_changed_are_looked_at_again():
    """Results whose elements come to lie in another order than their gradients' are refused, whichever
    of two lists that were used together has changed."""
    for which in (0, 1):
        ts, out = ([torch.randn(6, 10, device="cuda"), torch.randn(7, device="cuda")] for _ in range(2))
        g, o = ffi.GradList(ts), ffi.GradList(out)
        ws, stats = space(g), torch.empty(2, device="cuda")
        for _ in range(2):
            ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
        (ts, out)[which][0].data = torch.randn(10, 6, device="cuda").t()
        for _ in range(2):
            with pytest.raises(ValueError, match="result 0"):
                ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
        # Both in the same order again, though another one than before.
        (ts, out)[1 - which][0].data = torch.randn(10, 6, device="cuda").t()
        ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
        check(out, ts, 1.0, stats)


def test_lists_that_have_changed_in_place_are_looked_at_again():
    """The address and the number of elements as they were: another order is refused beside results of
    the first one, another type is read as what it is."""
    ts, out = ([torch.randn(6, 10, device="cuda"), torch.randn(7, device="cuda")] for _ in range(2))
    g, o = ffi.GradList(ts), ffi.GradList(out)
    ws, stats = space(g), torch.empty(2, device="cuda")
    for _ in range(2):
        ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
    for which in (ts, out):
        which[0].t_()
        for _ in range(2):
            with pytest.raises(ValueError, match="result 0"):
                ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
        which[0].t_()
        ffi.op_clip_gradients(g, 1.0, stats, out=o, workspace=ws)
        check(out, ts, 1.0, stats)
    buf = torch.randn(300, device="cuda")
    t = buf[:100]
    g = ffi.GradList([t])
    ws = space(g)
    ffi.op_clip_gradients(g, 1.0, stats, workspace=ws)
    buf.view(BF)[:100] = torch.randn(100, device="cuda").to(BF)
    t.data = buf.view(BF)[:100]
    before, rest = t.clone(), buf[50:].clone()
    ffi.op_clip_gradients(g, 0.5 * norm_of([before]), stats, workspace=ws)
    check([t], [before], 0.5 * norm_of([before]), stats)
    assert torch.equal(buf[50:], rest)
    t.data = buf[::2][:100]
    with pytest.raises(ValueError, match="one run"):
        ffi.op_clip_gradients(g, 1.0, stats, workspace=ws)


@pytest.mark.parametrize("size,limit", [(1e30, 1e-20), (1e30, 1e-9), (1e36, 1.0), (1e36, 1e-30), (1e30, 1e-42)])
def test_factors_below_the_range_of_fp32(size, limit):
    """limit / norm is subnormal or 0 in fp32; the results are not.  The factor in two parts: one rounding
    more in fp32 than a factor in range.  (Numbers below the smallest normal one are off by half of the smallest
    step, twice where they are rounded to bf16 after that.)"""
    sizes = [(4097, F32), (501, BF), (3, F32)]
    ts = tensors(sizes, offset=1, scale=size)
    ref, stats = norm_of(ts), torch.empty(2, device="cuda")
    out = tensors(sizes, seed=2, offset=2)
    ffi.op_clip_gradients(ts, limit, stats, out=out, workspace=space(ts))
    before = [t.clone() for t in ts]
    places = stats.tolist()
    ffi.op_clip_gradients(ts, limit, stats, workspace=space(ts))
    assert places == stats.tolist() and abs(places[0] - ref) <= 2.0 ** -23 * ref
    want = ctypes.c_float(limit).value / ref
    assert 0 < places[1] and abs(places[1] - want) <= 2.0 ** -149
    for t, o, was in zip(ts, out, before):
        assert torch.equal(t, o)
        w = was.double() * want
        step = torch.finfo(t.dtype).smallest_normal * torch.finfo(t.dtype).eps
        assert ((o.double() - w).abs() <= (torch.finfo(t.dtype).eps / 2 + 4 * 2.0 ** -24) * w.abs() + step).all()
        assert limit < 1e-37 or (o != 0).any()
