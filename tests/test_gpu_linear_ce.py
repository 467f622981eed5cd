"""Cross-entropy of a linear layer, its loss and gradients, against the formulas
in 64 bits.

Tolerances, with step = 2^-23 (one fp32 rounding or truncation, relative).  A
logit is a chain of dim + 1 sums: |error| <= E = (dim + 8) step S, S the sum of
the sizes of its terms.  The sum of exponentials adds at most classes / 16 + 256
roundings to a chain, and each exponent's argument one of at most its size:
lse is off by at most 2 E + (classes / 16 + 512 + 4 range + 4 |lse|) step =: F,
the loss by E more and four roundings of its parts.  A probability is then off by
a factor of exp(E + F + range step), and with q = p (E + F + (range + 8) step) the
gradient of a logit by w q and, where it is rounded, u |dz| (u = finfo(type).eps / 2;
fp32: one step).  dx and dW sum dz with |W| and |x| in chains of K = classes or rows
sums: |error| <= s (w q + u |dz|) |W| + (K + 8) step s |dz| |W| + u |dx|; dbias is
not rounded: s (w q + 2 step |dz|) summed, and (rows + 8) step of s |dz| summed.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
STEP = 2.0 ** -23
FILL = 7.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


def wide(t, pad):
    """A [rows, columns] tensor of t's values in a buffer with `pad` more columns."""
    buf = torch.full((t.shape[0], t.shape[1] + pad), FILL, dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


class Case:
    def __init__(self, dtype, rows, dim, classes, bias=False, weights=False, pad=0, spread=2.0, seed=0,
                 scale=0.37):
        g = torch.Generator().manual_seed(seed + rows + dim + classes)
        self.x = wide(torch.randn(rows, dim, generator=g).to(dtype).cuda(), pad)
        self.w = wide((torch.randn(classes, dim, generator=g) * spread / math.sqrt(dim)).to(dtype).cuda(), pad)
        self.b = torch.randn(classes, generator=g).cuda() if bias else None
        self.y = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32).cuda()
        self.rw = None
        if weights:
            self.rw = torch.tensor([0.0, 1.0, 0.25, -2.0])[torch.randint(0, 4, (rows,), generator=g)].cuda()
        self.scale, self.pad = scale, pad

    def space(self, backward):
        n = ffi.linear_cross_entropy_workspace(self.x, self.w, backward=backward)
        return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")   # NaN wherever it is read

    def forward(self, stream=None):
        r = self.x.shape[0]
        loss, lse = torch.full((r,), FILL, device="cuda"), torch.full((r,), FILL, device="cuda")
        ws = self.space(False)
        ffi.op_linear_cross_entropy(self.x, self.w, self.y, loss, bias=self.b, row_weight=self.rw,
                                    lse=lse, workspace=ws, stream=stream)
        return loss, lse

    def backward(self, lse, dx=True, dw=True, db=True):
        out = dict(dx=wide(torch.full_like(self.x, math.nan), self.pad) if dx else None,
                   dweight=wide(torch.full_like(self.w, math.nan), self.pad) if dw else None,
                   dbias=torch.full((self.w.shape[0],), math.nan, device="cuda") if db else None)
        ffi.op_linear_cross_entropy_bwd(self.x, self.w, self.y, lse, bias=self.b, row_weight=self.rw,
                                        scale=self.scale, workspace=self.space(True), **out)
        return out

    def reference(self):
        """{name: (value, tolerance)} in 64 bits, rows of weight 0 or bad labels left out."""
        x, w = self.x.double(), self.w.double()
        rows, dim = x.shape
        c = w.shape[0]
        wt = torch.ones(rows, dtype=torch.float64, device="cuda") if self.rw is None else self.rw.double()
        y = self.y.long()
        ok = (y >= 0) & (y < c)
        x = torch.where((wt != 0)[:, None], x, 0.0)
        b = torch.zeros(c, dtype=torch.float64, device="cuda") if self.b is None else self.b.double()
        z = x @ w.T + b
        size = x.abs() @ w.abs().T + torch.where(b.isinf(), 0.0, b.abs())
        e = (dim + 8) * STEP * size.amax(1)
        top = z.amax(1)
        seen = torch.where(z.isinf(), top[:, None], z)
        rng = top - seen.amin(1)
        lse = torch.logsumexp(z, 1)
        f = 2 * e + (c / 16 + 512 + 4 * rng + 4 * lse.abs()) * STEP
        zy = z.gather(1, y.clamp(0, c - 1)[:, None])[:, 0]
        none = wt == 0
        loss = torch.where(ok, lse - zy, math.nan).masked_fill(none, 0.0)
        tol = f + e + 4 * STEP * (zy.abs() + lse.abs())
        out = dict(loss=(loss, tol), lse=(lse.masked_fill(none, 0.0), f))
        p = torch.exp(z - lse[:, None])
        wt = torch.where(ok, wt, 0.0)
        dz = p.clone()
        dz[torch.arange(rows, device="cuda"), y.clamp(0, c - 1)] -= 1.0
        dz *= wt[:, None]
        q = wt.abs()[:, None] * p * (e + f + (rng + 8) * STEP)[:, None]
        u = torch.finfo(self.x.dtype).eps / 2 if self.x.dtype is BF else STEP
        s = abs(self.scale)
        err, mag = q + u * dz.abs(), dz.abs()
        dx, dw = self.scale * (dz @ w), self.scale * (dz.T @ x)
        out["dx"] = dx, s * ((err + (c + 8) * STEP * mag) @ w.abs()) + u * dx.abs()
        out["dweight"] = dw, s * ((err + (rows + 8) * STEP * mag).T @ x.abs()) + u * dw.abs()
        out["dbias"] = (self.scale * dz.sum(0),
                        s * (q + (2 + rows + 8) * STEP * mag).sum(0))
        return out


def holds(name, got, want):
    ref, tol = want
    bad = ~((got.double() - ref).abs() <= tol + 1e-37) & ~(got.isnan() & ref.isnan()) & ~(got.double() == ref)
    assert not bad.any(), (name, int(bad.sum()), got[bad][:4], ref[bad][:4], tol[bad][:4])


def check(case):
    ref = case.reference()
    loss, lse = case.forward()
    holds("loss", loss, ref["loss"])
    holds("lse", lse, ref["lse"])
    for n, t in case.backward(lse).items():
        holds(n, t, ref[n])
        if case.pad and t.dim() == 2:      # behind the rows nothing is written
            assert (torch.as_strided(t, (t.shape[0], case.pad), t.stride(), t.shape[1]) == FILL).all()


SIZES = [(1, 8, 1), (1, 64, 10), (3, 8, 2), (5, 40, 129), (64, 64, 64), (100, 72, 127), (129, 136, 300),
         (256, 768, 1000), (17, 384, 4099), (300, 64, 10007), (1000, 24, 33), (130, 1024, 257)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,classes", SIZES)
def test_loss_and_gradients(dtype, rows, dim, classes):
    check(Case(dtype, rows, dim, classes, bias=(rows + classes) % 2 == 0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,classes", [(70, 40, 200), (513, 128, 1000), (2, 16, 5)])
def test_weights_of_rows_and_strides(dtype, rows, dim, classes):
    check(Case(dtype, rows, dim, classes, bias=True, weights=True, pad=24))


def test_odd_dimensions_of_fp32():
    check(Case(F32, 40, 12, 100))
    check(Case(F32, 40, 100, 65, pad=4))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_rows_take_pieces(dtype):
    """More classes than one piece of the backward pass holds."""
    case = Case(dtype, 70000, 16, 4500, weights=True, bias=True)
    check(case)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_left_out_may_hold_anything(dtype):
    case = Case(dtype, 300, 64, 500, weights=True, bias=True)
    ref = case.reference()
    case.x[case.rw == 0] = math.nan
    case.y[case.rw == 0] = -7
    loss, lse = case.forward()
    holds("loss", loss, ref["loss"])
    for n, t in case.backward(lse).items():
        holds(n, t, ref[n])
    assert (case.backward(lse)["dx"][case.rw == 0] == 0).all()


# Sizes at which rows of weight 0 are set aside before the products (over 4e10 operations, fp32 ones
# counted eight times); 300000 rows are too many for it.
GATHERED = [(BF, 1000, 512, 41003), (F32, 1000, 256, 10007), (BF, 70000, 16, 20000), (F32, 20000, 16, 8200),
            (BF, 300000, 32, 2100)]


@pytest.mark.parametrize("dtype,rows,dim,classes", GATHERED)
def test_rows_are_set_aside(dtype, rows, dim, classes):
    case = Case(dtype, rows, dim, classes, weights=True, bias=True, pad=16)
    case.y[::7] = -1
    ref = case.reference()
    case.x[case.rw == 0] = math.nan
    loss, lse = case.forward()
    holds("loss", loss, ref["loss"])
    holds("lse", lse, ref["lse"])
    got = case.backward(lse)
    for n, t in got.items():
        holds(n, t, ref[n])
    assert (got["dx"][(case.rw == 0) | (case.y < 0)] == 0).all()
    again = case.backward(lse)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("share", [0.0, 0.002, 1.0])
def test_all_or_hardly_any_rows_count(share):
    case = Case(BF, 1000, 512, 41003, bias=True)
    g = torch.Generator().manual_seed(3)
    case.rw = (torch.rand(1000, generator=g) < share).float().cuda()
    ref = case.reference()
    loss, lse = case.forward()
    holds("loss", loss, ref["loss"])
    for n, t in case.backward(lse).items():
        holds(n, t, ref[n])
        assert share > 0 or (t == 0).all()
    only = case.backward(lse, dx=False, dw=False)
    assert torch.equal(only["dbias"], case.backward(lse)["dbias"])


def test_setting_rows_aside_is_captured():
    case = Case(BF, 1000, 512, 41003, weights=True)
    loss, lse = torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    dx, dw = torch.empty_like(case.x), torch.empty_like(case.w)
    wf, wb = case.space(False), case.space(True)

    def step():
        ffi.op_linear_cross_entropy(case.x, case.w, case.y, loss, row_weight=case.rw, lse=lse, workspace=wf)
        ffi.op_linear_cross_entropy_bwd(case.x, case.w, case.y, lse, dx=dx, dweight=dw, row_weight=case.rw,
                                        workspace=wb)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for i in range(3):   # other rows count at each replay
        case.rw.copy_(torch.randint(0, 2, (1000,), generator=torch.Generator().manual_seed(i)).float())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, lse, dx, dw)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, lse, dx, dw)))
        assert int((loss == 0).sum()) >= int((case.rw == 0).sum()) > 300


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bad_labels_make_their_loss_nan_and_nothing_else(dtype):
    case = Case(dtype, 50, 32, 70)
    case.y[3], case.y[20], case.y[49] = -1, 70, 2 ** 31 - 1
    ref = case.reference()
    loss, lse = case.forward()
    assert loss[[3, 20, 49]].isnan().all() and int(loss.isnan().sum()) == 3
    holds("lse", lse, ref["lse"])
    for n, t in case.backward(lse).items():
        holds(n, t, ref[n])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_classes_left_out_by_the_bias(dtype):
    case = Case(dtype, 60, 64, 400, bias=True)
    case.b[128:390] = -math.inf          # whole tiles, and parts of them
    case.y.clamp_(max=127)
    check(case)
    loss, lse = case.forward()
    got = case.backward(lse)
    assert (got["dweight"][128:390] == 0).all() and (got["dbias"][128:390] == 0).all()


def test_a_label_that_the_bias_leaves_out_costs_infinitely_much():
    case = Case(F32, 4, 16, 30, bias=True)
    case.b[5] = -math.inf
    case.y[:] = torch.tensor([5, 6, 5, 7])
    loss, _ = case.forward()
    assert loss[[0, 2]].isinf().all() and (loss[[0, 2]] > 0).all() and loss[[1, 3]].isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_logits(dtype):
    """Logits in the thousands: the largest takes all."""
    check(Case(dtype, 40, 64, 300, spread=800.0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_each_gradient_by_itself(dtype):
    case = Case(dtype, 90, 48, 310, bias=True, weights=True)
    _, lse = case.forward()
    both = case.backward(lse)
    for n, one in (("dx", case.backward(lse, True, False, False)), ("dweight", case.backward(lse, False, True, False)),
                   ("dbias", case.backward(lse, False, False, True))):
        assert torch.equal(one[n], both[n])


def test_no_rows():
    case = Case(F32, 0, 16, 30, bias=True)
    loss, lse = case.forward()
    got = case.backward(lse)
    assert loss.numel() == 0 and (got["dweight"] == 0).all() and (got["dbias"] == 0).all()


def test_gradients_against_differences():
    """The loss moves as the gradient says when W moves by t D to either side: up to the third
    derivative (at most the logits' largest change cubed, over 6, times 2), and the two losses' own
    errors over 2 t."""
    case = Case(F32, 30, 32, 50, scale=1.0)
    ref = case.reference()
    loss, lse = case.forward()
    got = case.backward(lse)
    g = torch.Generator().manual_seed(3)
    d = torch.randn(50, 32, generator=g).cuda()
    t = 2.0 ** -10
    w0 = case.w.clone()
    sums = []
    for sign in (1, -1):
        case.w.copy_(w0 + sign * t * d)
        sums.append(case.forward()[0].double().sum())
    moved = (sums[0] - sums[1]) / (2 * t)
    said = (got["dweight"].double() * d.double()).sum()
    third = (t ** 2) * ((d.double() @ case.x.double().T).abs().amax(0) ** 3).sum()
    # w0 +- t d are rounded to fp32: off by 2^-24 |w| each, which moves a logit by that times |x|.
    rounding = (2 * ref["loss"][1].sum() + 2.0 ** -23 * (w0.abs().double() @ case.x.abs().double().T).amax(0).sum()) / (2 * t)
    assert abs(moved - said) <= third + rounding


def test_same_bits_every_time_and_on_another_stream():
    case = Case(BF, 400, 256, 5000, bias=True, weights=True)
    loss, lse = case.forward()
    first = case.backward(lse)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        loss2, lse2 = case.forward()
        second = case.backward(lse2)
    s.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    for n in first:
        assert torch.equal(first[n], second[n])


def test_captured_and_replayed():
    case = Case(BF, 200, 64, 1000, bias=True, weights=True)
    loss, lse = torch.empty(200, device="cuda"), torch.empty(200, device="cuda")
    dx, dw, db = torch.empty_like(case.x), torch.empty_like(case.w), torch.empty_like(case.b)
    wf, wb = case.space(False), case.space(True)

    def step():
        ffi.op_linear_cross_entropy(case.x, case.w, case.y, loss, bias=case.b, row_weight=case.rw, lse=lse,
                                    workspace=wf)
        ffi.op_linear_cross_entropy_bwd(case.x, case.w, case.y, lse, dx=dx, dweight=dw, dbias=db, bias=case.b,
                                        row_weight=case.rw, scale=0.1, workspace=wb)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for i in range(4):
        with torch.no_grad():
            case.x.copy_(torch.randn(200, 64, generator=torch.Generator().manual_seed(i)).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, lse, dx, dw, db)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (loss, lse, dx, dw, db)):
            assert torch.equal(a, b)
