"""The largest logits of each row and the distillation loss on them, against the
formulas in 64 bits.

Largest logits: whole numbers and copied values, so equal.

Distillation tolerances, e = 2^-24.  An exponential in base 2 of an argument of
size A is within (2 A + 4) e of itself, relative (A rounded, times a factor,
then the instruction's one ulp); A is at most 1.45 spread / temperature, spread
the largest distance of a logit from the row's maximum that still counts (at
most 104 in base 2: beyond it the term is under 2^-104).  A sum of C terms by
512 or 1024 threads adds (C / 512 + 32) e.  Call d the total; with temperature
tau, the loss is within
  alpha tau^2 (4 d + 8 e sum p (|log p| + |log q|)) + (1 - alpha) (2 d + 8 e |lse - z|),
and a gradient within u |g| + w (alpha tau (q + p) + (1 - alpha) (q1 + [label]))
(2 d + 16 e), u = finfo(type).eps / 2 for its rounding.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FILL = 7.0
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


# ------------------------------------------------------------------- largest logits

def top_ref(z, top):
    """Largest first, the lower index first among equal ones, NaN above all."""
    key = torch.where(torch.isnan(z), math.inf, z.double())
    nan = torch.isnan(z)
    order = torch.argsort(-key, dim=1, stable=True)
    order = torch.cat([torch.cat([r[n[r]], r[~n[r]]])[None] for r, n in zip(order, nan)])
    return order[:, :top]


def check_top(z, top):
    values = torch.full((z.shape[0], top), FILL, device="cuda")
    indices = torch.full((z.shape[0], top), -7, dtype=torch.int32, device="cuda")
    ffi.op_top_logits(z, values, indices)
    want = top_ref(z.cpu(), top)
    assert torch.equal(indices.cpu().long(), want)
    got, ref = values.cpu(), z.cpu().float().gather(1, want)
    assert torch.equal(torch.nan_to_num(got, nan=1e38), torch.nan_to_num(ref, nan=1e38))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,classes,top", [
    (1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 256, 256), (64, 1000, 16), (3, 999, 1), (2, 2047, 256),
    (2, 2049, 255), (2, 8191, 100), (2, 8192, 256), (3, 8193, 64), (2, 33333, 7), (2, 131072, 256),
    (1, 200003, 64)])
def test_top_logits(dtype, rows, classes, top):
    g = torch.Generator().manual_seed(classes + top)
    check_top((torch.randn(rows, classes, generator=g) * 3).to(dtype).cuda(), top)


@pytest.mark.parametrize("classes", [64, 65, 422, 512, 513, 2048, 2049, 4096, 4097, 8191])
@pytest.mark.parametrize("top", [1, 54, 56, 57, 64, 129, 224, 225, 256])
def test_top_logits_of_few_classes(classes, top):
    """bf16 values, many of them equal: where one wave, four or eight take a row, read one by one
    or in runs, and the last keys fit a wave or do not."""
    g = torch.Generator().manual_seed(classes * 257 + top)
    check_top(torch.randn(9, classes, generator=g).to(BF).cuda(), min(top, classes))


@pytest.mark.parametrize("classes", [300, 9001, 70000])
@pytest.mark.parametrize("kind", ["equal", "two", "rising", "falling", "one share", "infinite",
                                  "nan", "zeros"])
def test_top_logits_of_awkward_rows(kind, classes):
    """Ties everywhere; the largest values in few threads' shares (more keys than are held at
    once); infinities, NaN and both zeros."""
    i = torch.arange(classes)
    g = torch.Generator().manual_seed(1)
    z = torch.randn(classes, generator=g)
    if kind == "equal":
        z = torch.full((classes,), -2.5)
    elif kind == "two":
        z = (i * 7 % 3 == 0).float()
    elif kind == "rising":
        z = i.float()
    elif kind == "falling":
        z = -i.float()
    elif kind == "one share":
        z[(i // 8) % 256 < 16] += 100
        z[(i // 8) % 1024 < 3] += 100
    elif kind == "infinite":
        z[::3] = -math.inf
        z[5::97] = math.inf
    elif kind == "nan":
        z[11::50] = math.nan
        z[7] = -math.nan
    elif kind == "zeros":
        z = torch.where(i % 2 == 0, -0.0, 0.0)
    for top in (1, 20, 256):
        check_top(torch.stack([z, z.flip(0)]).cuda(), min(top, classes))


def test_top_logits_rows_of_any_stride_and_alignment():
    g = torch.Generator().manual_seed(2)
    for dtype in (BF, F32):
        buf = torch.randn(6, 1037, generator=g).to(dtype).cuda()
        for a in range(0, 9):
            check_top(buf[1:5, a:a + 1001], 9)


def test_top_logits_captured():
    g = torch.Generator().manual_seed(4)
    z = torch.randn(40, 20000, generator=g).cuda()
    v, i = torch.empty(40, 8, device="cuda"), torch.empty(40, 8, dtype=torch.int32, device="cuda")
    ffi.op_top_logits(z, v, i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffi.op_top_logits(z, v, i)
    for _ in range(3):
        z.copy_(torch.randn(40, 20000, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(i.cpu().long(), top_ref(z.cpu(), 8))


# --------------------------------------------------------------------- distillation

class Distill:
    def __init__(self, dtype=F32, grad=F32, rows=3, classes=100, top=8, tau=2.0, alpha=0.5,
                 labels=True, weight=None, scale=1.0, gain=3.0, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed + classes * 3 + top)
        self.rows, self.c, self.top, self.tau, self.alpha = rows, classes, top, tau, alpha
        self.scale, self.grad = scale, grad
        buf = (torch.randn(rows, classes + pad, generator=g) * gain).to(dtype).cuda()
        self.z = buf[:, pad:] if pad else buf
        self.idx = torch.stack([torch.randperm(classes, generator=g)[:top] for _ in range(rows)]) \
            .to(torch.int32).cuda()
        self.val = (torch.randn(rows, top, generator=g) * 2 + 5).cuda()
        self.y = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32).cuda() \
            if labels else None
        self.w = None if weight is None else torch.tensor(weight, dtype=F32).cuda()

    def run(self, grad=True, into=None):
        loss = torch.full((self.rows,), FILL, device="cuda")
        d = into
        if grad and d is None:
            d = torch.full((self.rows, self.c), FILL, dtype=self.grad, device="cuda")
        ffi.op_distill(self.z, self.val if self.top else None, self.idx if self.top else None, loss,
                       dlogits=d, labels=self.y, temperature=self.tau, alpha=self.alpha,
                       row_weight=self.w, scale=self.scale)
        return loss, d

    def reference(self):
        z, tau, a = self.z.double().cpu(), self.tau, self.alpha
        idx, val = self.idx.long().cpu(), self.val.double().cpu()
        loss, lt = torch.zeros(self.rows).double(), torch.zeros(self.rows).double()
        grad, gt = torch.zeros_like(z), torch.zeros_like(z)
        for r in range(self.rows):
            w = 1.0 if self.w is None else self.w[r].item()
            if w == 0:
                continue
            zr = z[r]
            spread = min(104.0, 1.45 * (zr.max() - zr[zr > -math.inf].min()).item() / min(tau, 1.0))
            d = (2 * spread + 4 + self.c / 512 + 32) * E
            on = idx[r] >= 0
            if a > 0 and on.any() and (val[r][on] > -math.inf).any():
                lp = torch.log_softmax(val[r][on] / tau, 0)
                lq_all = torch.log_softmax(zr / tau, 0)
                p, lq = lp.exp(), lq_all[idx[r][on]]
                terms = torch.where(p > 0, p * (lp - lq), 0.0)
                loss[r] += a * tau * tau * terms.sum()
                lt[r] += a * tau * tau * (4 * d + 8 * E * torch.where(
                    p > 0, p * (lp.abs() + lq.abs()), 0.0).sum())
                at = torch.zeros_like(zr).index_add_(0, idx[r][on], p)
                grad[r] += a * tau * (lq_all.exp() - at)
                gt[r] += a * tau * (lq_all.exp() + at)
            if self.y is not None and a < 1:
                l1 = torch.log_softmax(zr, 0)
                y = int(self.y[r])
                loss[r] -= (1 - a) * l1[y]
                lt[r] += (1 - a) * (2 * d + 8 * E * l1[y].abs())
                hot = torch.zeros_like(zr)
                hot[y] = 1
                grad[r] += (1 - a) * (l1.exp() - hot)
                gt[r] += (1 - a) * (l1.exp() + hot)
            grad[r] *= w * self.scale
            gt[r] *= abs(w * self.scale) * (2 * d + 16 * E)
        return loss, lt, grad, gt

    def check(self, loss, grad):
        ref, lt, gref, gt = self.reference()
        err = (loss.double().cpu() - ref).abs()
        assert ((err <= lt) | (loss.cpu() == ref)).all(), (err, lt)
        if grad is None:
            return
        u = torch.finfo(grad.dtype).eps / 2
        gerr = (grad.double().cpu() - gref).abs()
        # Results under the type's smallest normal number are rounded to its steps there.
        tiny = torch.finfo(grad.dtype).tiny
        assert (gerr <= gt + u * gref.abs() + tiny).all(), (gerr - gt).max()


CASES = [
    dict(),
    dict(dtype=BF, grad=BF),
    dict(dtype=BF, grad=F32, tau=1.0),
    dict(grad=BF, tau=4.0, alpha=0.9, classes=1000, top=16, rows=5),
    dict(alpha=1.0, labels=False),
    dict(alpha=1.0, labels=True),
    dict(alpha=0.0, top=0),
    dict(alpha=0.0, top=4, tau=3.0),
    dict(classes=1, top=1),
    dict(classes=7, top=7, tau=0.25),
    dict(classes=9, top=2, rows=1, pad=3, dtype=BF, grad=BF),
    dict(classes=511, top=256, pad=1, dtype=BF, grad=F32),
    dict(classes=8191, top=33, tau=1.0, alpha=1.0, labels=False, dtype=BF, grad=BF),
    dict(classes=8192, top=64, dtype=BF, grad=BF, tau=1.5),
    dict(classes=50021, top=32, rows=2, pad=5),
    dict(classes=131072, top=256, rows=2, dtype=BF, grad=BF),
    dict(classes=200003, top=3, rows=1, tau=8.0, grad=BF),
    dict(weight=[0.0, 2.5, -1.0], scale=0.125),
    dict(gain=80.0, tau=1.0),
    dict(gain=0.0),
]


@pytest.mark.parametrize("kw", CASES, ids=str)
def test_distill(kw):
    c = Distill(**kw)
    loss, grad = c.run()
    c.check(loss, grad)
    alone, _ = c.run(grad=False)
    assert torch.equal(alone, loss)


@pytest.mark.parametrize("dtype,classes", [(BF, 110000), (BF, 179200), (BF, 179203), (F32, 60001),
                                           (F32, 89600), (F32, 89603)])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distill_long_rows_at_one_and_two_temperatures(dtype, classes, tau):
    """To either side of the lengths from which a workgroup has more threads."""
    c = Distill(dtype=dtype, grad=dtype, rows=2, classes=classes, top=40, tau=tau)
    loss, grad = c.run()
    c.check(loss, grad)
    assert torch.equal(c.run(grad=False)[0], loss)


@pytest.mark.parametrize("dtype,classes", [(F32, 300), (BF, 9001)])
def test_distill_over_its_own_logits(dtype, classes):
    c = Distill(dtype=dtype, grad=dtype, classes=classes)
    loss, grad = c.run()
    l2, g2 = c.run(into=c.z)
    assert torch.equal(loss, l2) and torch.equal(grad, g2)


def test_distill_same_class_twice_and_as_label():
    c = Distill(classes=50, top=6)
    c.idx[0] = torch.tensor([3, 9, 3, 3, 9, 40])
    c.idx[1] = 17
    c.y[0], c.y[1] = 3, 17
    c.check(*c.run())


def test_distill_rows_with_few_or_no_entries():
    c = Distill(rows=4, classes=60, top=5)
    c.idx[0, 2:] = -1
    c.idx[1] = -1
    c.val[1] = math.nan                              # not there: not looked at
    c.val[2] = -math.inf
    c.val[3, :4] = -math.inf
    c.check(*c.run())
    c = Distill(rows=4, classes=60, top=5, alpha=1.0, labels=False)
    c.idx[0, 1:] = -1
    c.idx[1] = -1
    loss, grad = c.run()
    c.check(loss, grad)
    assert loss[1] == 0 and (grad[1] == 0).all()


def test_distill_row_of_weight_zero_is_not_read():
    c = Distill(rows=3, classes=9000, dtype=BF, grad=BF, weight=[1.0, 0.0, 1.0])
    c.z[1] = math.nan
    c.idx[1] = 1 << 30
    c.y[1] = -5
    loss, grad = c.run()
    assert loss[1] == 0 and (grad[1] == 0).all()
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("classes", [40, 10000])
def test_distill_bad_classes_make_the_loss_nan(classes):
    c = Distill(rows=5, classes=classes)
    good, _ = c.run()
    c.idx[0, 1], c.idx[1, 2] = classes, -2
    c.y[2], c.y[3] = classes, -1
    loss, grad = c.run()
    assert torch.isnan(loss[:4]).all() and loss[4] == good[4]
    assert torch.isfinite(grad).all()


def test_distill_infinite_logits():
    """-infinity is a class that cannot be: no weight, no gradient, and an infinite loss where the
    teacher wants it.  NaN and +infinity spread over their row only."""
    c = Distill(rows=4, classes=64, top=4, alpha=1.0, labels=False)
    free = [i for i in range(64) if i not in c.idx[0].tolist()]
    c.z[0, free[:9]] = -math.inf
    c.z[1, c.idx[1, 0].long()] = -math.inf
    c.z[2, 5] = math.nan
    c.z[3, 5] = math.inf
    loss, grad = c.run()
    assert torch.isfinite(loss[0]) and (grad[0, free[:9]] == 0).all()
    assert loss[1] == math.inf and torch.isfinite(grad[1]).all()
    assert torch.isnan(loss[2:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("classes", [200, 9003])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_distill_masks_of_the_lowest_value(dtype, classes, tau):
    """Classes masked by the type's lowest finite value have no weight; a row of nothing else is
    uniform.  Far out, only logits equal to the maximum count."""
    low = torch.finfo(dtype).min
    c = Distill(dtype=dtype, grad=F32, rows=5, classes=classes, top=4, tau=tau)
    c.idx[:], c.y[:] = torch.tensor([1, 3, 5, 7], dtype=torch.int32), 3
    c.z[0, 8:] = low
    c.z[1] = low                                       # nothing is left
    c.z[2], c.z[2, 1:9:2] = 1.0e30, 2.0e30             # the teacher's classes are the largest
    c.z[3], c.z[3, 1:9:2] = low, -1.0e30
    c.val[4, :] = torch.finfo(F32).min                 # a teacher without an opinion
    c.val[0, 1:] = torch.finfo(F32).min
    loss, grad = c.run()
    c.check(loss, grad)
    assert torch.isfinite(loss).all() and (grad[0, 9:] == 0).all()


def test_distill_label_on_a_masked_class():
    """Its loss is the distance, finite as long as that is."""
    c = Distill(classes=70, top=0, alpha=0.0)
    c.z[:, 11], c.y[:] = -1.0e38, 11
    c.check(*c.run())


@pytest.mark.parametrize("grad,pad", [(BF, 0), (BF, 3), (F32, 1)])
def test_distill_rows_left_out_are_filled_with_zeros(grad, pad):
    """... whole, at any alignment, and nothing beside them is written."""
    c = Distill(rows=3, classes=1003, weight=[0.0, 0.0, 1.0])
    buf = torch.full((3, 1003 + 8), FILL, dtype=grad, device="cuda")
    into = buf[:, pad:pad + 1003]
    c.run(into=into)
    assert (into[:2] == 0).all() and (into[2] != FILL).all()
    assert (buf[:, :pad] == FILL).all() and (buf[:, pad + 1003:] == FILL).all()


def test_distill_gradient_against_differences():
    """h = 2^-6: truncation ~ h^2 / 6 of a third derivative near 1, rounding ~ 8 * 2^-24 loss / h."""
    c = Distill(rows=1, classes=30, top=5, gain=1.0, tau=1.5)
    _, grad = c.run()
    h = 2.0 ** -6
    for j in [int(c.idx[0, 0]), int(c.y[0]), 4, 29]:
        z0 = c.z[0, j].item()
        f = []
        for s in (h, -h):
            c.z[0, j] = z0 + s
            f.append(c.run()[0].item())
        c.z[0, j] = z0
        assert abs((f[0] - f[1]) / (2 * h) - grad[0, j].item()) < 5e-4


def test_distill_captured_and_on_another_stream():
    c = Distill(rows=20, classes=9001, dtype=BF, grad=BF, top=16)
    g = torch.Generator().manual_seed(8)
    loss = torch.empty(20, device="cuda")
    grad = torch.empty(20, 9001, dtype=BF, device="cuda")

    def step():
        ffi.op_distill(c.z, c.val, c.idx, loss, dlogits=grad, labels=c.y, temperature=c.tau,
                       alpha=c.alpha)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        c.z.copy_(torch.randn(20, 9001, generator=g).to(BF))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            l2, g2 = c.run()
        side.synchronize()
        loss.fill_(FILL)
        grad.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, l2) and torch.equal(grad, g2)


def test_more_rows_than_one_launch_holds():
    """2^21 rows and a few: the largest logits are copies, equal to a sort's; of the loss
    the last rows are those of a call for them alone, bit for bit."""
    rows, n = (1 << 21) + 5, 100
    g = torch.Generator(device="cuda").manual_seed(5)
    z = torch.randn(rows, 10, device="cuda", generator=g)
    values = torch.full((rows, 2), FILL, device="cuda")
    indices = torch.full((rows, 2), -7, dtype=torch.int32, device="cuda")
    ffi.op_top_logits(z, values, indices)
    assert torch.equal(values, torch.topk(z, 2, dim=1).values)
    assert torch.equal(values, z.gather(1, indices.long())) and (indices[:, 0] != indices[:, 1]).all()
    y = indices[:, 1].contiguous()
    loss, grad = torch.full((rows,), FILL, device="cuda"), torch.full_like(z, FILL)
    ffi.op_distill(z, values, indices, loss, dlogits=grad, labels=y, temperature=2.0, alpha=0.5)
    some, sgrad = torch.empty(n, device="cuda"), torch.empty(n, 10, device="cuda")
    for at in (0, rows - n):
        ffi.op_distill(z[at:at + n], values[at:at + n], indices[at:at + n], some, dlogits=sgrad,
                       labels=y[at:at + n], temperature=2.0, alpha=0.5)
        assert torch.equal(some, loss[at:at + n]) and torch.equal(sgrad, grad[at:at + n])
    assert (loss != FILL).all() and torch.isfinite(loss).all()
