"""A training step's operators on tensors that reach far: gradients beyond the caches, which the
clipping reads past them, and rows more than 2^32 bytes behind the first.  Tolerances: those of the
operators' own tests."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402
import test_gpu_block_norm as bn  # noqa: E402
import test_gpu_clip as clip  # noqa: E402
import test_gpu_linear_ce as ce  # noqa: E402
import test_gpu_qk_axes as axes  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("offset", [0, 1])
def test_clipping_of_more_than_the_caches_hold(offset):
    """400 MB of both types: the launches that pass the caches by, in place and beside."""
    ts = clip.tensors([(70_000_003, F32), (17, BF), (60_000_008, BF), (5, F32)], offset=offset)
    ref = clip.norm_of(ts)
    stats = torch.empty(2, device="cuda")
    out = [torch.full_like(t, math.nan) for t in ts]
    ffi.op_clip_gradients(ts, 0.3 * ref, stats, out=out, workspace=clip.space(ts))
    clip.check(out, ts, 0.3 * ref, stats)
    before = [t.clone() for t in ts]
    ffi.op_clip_gradients(ts, 0.3 * ref, stats, workspace=clip.space(ts))
    clip.check(ts, before, 0.3 * ref, stats)
    for t, o in zip(ts, out):
        assert torch.equal(t, o)
    for t in ts:
        edge = t._base
        at = t.storage_offset()
        assert edge[:at].isnan().all() and edge[at + t.numel():].isnan().all()


def spread(shape, strides, dtype, places):
    """`places` tensors side by side in one buffer with these strides; the buffer is not touched."""
    n = sum((s - 1) * st for s, st in zip(shape, strides)) + places * shape[-1]
    buf = torch.empty(n, dtype=dtype, device="cuda")
    return [torch.as_strided(buf, shape, strides, i * shape[-1]) for i in range(places)]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear_cross_entropy_of_rows_far_apart(dtype):
    rows, dim, classes, ld = 2600, 64, 2500, 1 << 20    # 5 and 10 GB
    c = ce.Case(dtype, rows, dim, classes, bias=True, weights=True)
    ref = c.reference()
    x, dx = spread((rows, dim), (ld, 1), dtype, 2)
    w, dw = spread((classes, dim), (ld, 1), dtype, 2)
    x.copy_(c.x)
    w.copy_(c.w)
    c.x, c.w = x, w
    loss, lse = c.forward()
    ce.holds("loss", loss, ref["loss"])
    ce.holds("lse", lse, ref["lse"])
    ffi.op_linear_cross_entropy_bwd(x, w, c.y, lse, dx=dx, dweight=dw, bias=c.b, row_weight=c.rw, scale=c.scale,
                                    workspace=c.space(True))
    ce.holds("dx", dx, ref["dx"])
    ce.holds("dweight", dw, ref["dweight"])


@pytest.mark.parametrize("d", [40, 1100, 8300])
def test_block_norm_of_tokens_far_apart(d):
    b, t = 2, 3
    c = bn.Case(BF, BF, b, t, d, kind="layer", gate="sequence")
    strides = (3 << 30, 1 << 30, 1)      # elements of 2 bytes: 6 GB to the second sequence
    x, y, dx_out, du, out, u = spread((b, t, d), strides, BF, 6)
    for far, near in ((x, c.x), (y, c.y), (dx_out, c.dx_out), (du, c.du)):
        far.copy_(near)
    c.x, c.y, c.dx_out, c.du = x, y, dx_out, du
    ffi.op_block_norm(x, y, out, u, **c.kw)
    c.check_forward(out.contiguous(), u.contiguous())
    c.empty = lambda dtype: {0: out, 1: u}[c.__dict__.setdefault("turn", iter((0, 1))).__next__()]
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotation_of_tokens_far_apart(dtype):
    c = axes.Axes(dtype, 2, 3, 2, 1, 64, (12, 20))
    strides = (3 << 30, 1 << 30, 64, 1)
    for n in "qk":
        h = c.heads[n]
        buf = torch.empty((5 << 30) + 2 * h * 64, dtype=dtype, device="cuda")
        far = torch.as_strided(buf, (2, 3, h, 64), strides)
        far.copy_(c.x[n])
        c.x[n] = far
    c.check_forward(c.forward())
    c.check_backward(*c.backward())
