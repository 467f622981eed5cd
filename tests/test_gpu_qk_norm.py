"""Per-head norms of q and k with the position rotation, forward and backward,
against the formulas in 64 bits.

Tolerances.  One rounding to the result's type is off by at most half a step,
u = finfo(type).eps / 2 relative.  Before it a result is a c - b s with a and b
each within a few fp32 roundings (the mean of squares: dim of them, but it
enters through its square root and a tree of sums): |error| <= u |result| +
64 * 2^-24 (|a| + |b|).  dx likewise, with |g| + |u mean(g u)| in the place of
|a| + |b| (g itself one rotation).  A weight gradient sums n terms in fp32:
(n / 64 + 64) * 2^-24 of the sum of their sizes covers the longest chain (a lane
walks at most n / 64 of them).
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FILL = 7.0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


def turn(y, c, s, rot, pairs):
    """(y rotated, |a| + |b| of each result) in 64 bits; c, s: [..., rot / 2]."""
    out, size = y.clone(), y.abs()
    if rot:
        lo = slice(0, rot, 2) if pairs else slice(0, rot // 2)
        hi = slice(1, rot, 2) if pairs else slice(rot // 2, rot)
        a, b = y[..., lo], y[..., hi]
        out[..., lo], out[..., hi] = a * c - b * s, b * c + a * s
        size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return out, size


class Case:
    def __init__(self, dtype, b, t, h, kv, dim, rot, pairs=False, layout="plain", lens=None,
                 positions=True, gamma=True, seed=0):
        g = torch.Generator().manual_seed(seed + dim + t)
        self.dtype, self.b, self.t, self.dim, self.rot, self.pairs = dtype, b, t, dim, rot, pairs
        self.heads = {"q": h, "k": kv}
        if layout == "packed":                 # [b][t][head][q k v][dim]
            buf = torch.randn(b, t, h, 3, dim, generator=g).to(dtype).cuda()
            self.x = {"q": buf[:, :, :, 0], "k": buf[:, :, :, 1]}
        elif layout == "cache":                # [b][head][capacity][dim], tokens in the middle
            self.x = {n: torch.randn(b, m, t + 5, dim, generator=g).to(dtype).cuda()
                      .transpose(1, 2)[:, 2:2 + t] for n, m in self.heads.items()}
        else:
            self.x = {n: (torch.randn(b, t, m, dim, generator=g) * 1.5).to(dtype).cuda()
                      for n, m in self.heads.items()}
        self.gamma = {n: (1 + 0.3 * torch.randn(dim, generator=g)).cuda() if gamma else None
                      for n in "qk"}
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
        rows = t + 40
        self.positions = (torch.randint(0, rows, (b, t), generator=g, dtype=torch.int32).cuda()
                          if positions and rot else None)
        ang = torch.rand(rows, max(rot // 2, 1), generator=g, dtype=torch.float64) * 100
        self.cos, self.sin = ((ang.cos().float().cuda(), ang.sin().float().cuda()) if rot
                              else (None, None))
        self.eps = 1e-5
        self.kw = dict(cos=self.cos, sin=self.sin, q_gamma=self.gamma["q"], k_gamma=self.gamma["k"],
                       positions=self.positions, lens=self.lens, eps=self.eps, interleaved=pairs)

    def tables(self):
        if not self.rot:
            return None, None
        pos = (self.positions.long() if self.positions is not None else
               torch.arange(self.t, device="cuda")[None].expand(self.b, self.t))
        return self.cos.double()[pos][:, :, None], self.sin.double()[pos][:, :, None]

    def inside(self):
        m = torch.ones(self.b, self.t, dtype=torch.bool, device="cuda")
        if self.lens is not None:
            m = torch.arange(self.t, device="cuda")[None] < self.lens[:, None]
        return m

    def empty(self, n):
        return torch.full((self.b, self.t, self.heads[n], self.dim), FILL, dtype=self.dtype,
                          device="cuda")

    def norm(self, n):
        x = self.x[n].double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + self.eps)
        w = self.gamma[n].double() if self.gamma[n] is not None else torch.ones_like(x[0, 0, 0])
        return x * r, r, w

    def check_forward(self, out):
        u = torch.finfo(self.dtype).eps / 2
        c, s = self.tables()
        m = self.inside()
        for n in "qk":
            if not self.heads[n]:
                continue
            un, _, w = self.norm(n)
            ref, size = turn(un * w, c, s, self.rot, self.pairs)
            got = out[n].double()
            tol = u * ref.abs() + 64 * 2.0 ** -24 * size
            assert ((got - ref).abs() <= tol)[m].all(), (n, (got - ref).abs()[m].max().item())
            assert (got[~m] == FILL).all(), "rows behind a sequence were written"


CASES = [
    # dtype, batch, tokens, q heads, k heads, dim, rot, pairs, layout
    (BF, 2, 7, 3, 3, 64, 64, False, "packed"),
    (BF, 1, 1, 12, 12, 64, 64, False, "packed"),
    (BF, 3, 197, 6, 2, 128, 96, True, "plain"),
    (BF, 2, 33, 5, 1, 80, 48, False, "plain"),
    (BF, 2, 9, 4, 4, 96, 96, True, "cache"),
    (BF, 1, 70, 8, 2, 256, 128, False, "cache"),
    (BF, 2, 5, 1, 1, 16, 16, False, "plain"),
    (BF, 2, 5, 3, 2, 32, 0, False, "plain"),
    (F32, 2, 7, 3, 3, 64, 64, False, "packed"),
    (F32, 1, 61, 5, 1, 80, 48, True, "plain"),
    (F32, 2, 19, 4, 2, 128, 128, False, "cache"),
    (F32, 1, 3, 2, 1, 256, 256, False, "plain"),
    (F32, 4, 1, 1, 1, 16, 16, True, "plain"),
]


@pytest.mark.parametrize("args", CASES, ids=str)
def test_forward(args):
    c = Case(*args[:7], pairs=args[7], layout=args[8])
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    c.check_forward(out)


def backward(c, seed=5, weights=True):
    g = torch.Generator().manual_seed(seed)
    d = {n: torch.randn(c.b, c.t, c.heads[n], c.dim, generator=g).to(c.dtype).cuda() for n in "qk"}
    dx = {n: c.empty(n) for n in "qk"}
    dw = {n: torch.full((c.dim,), FILL, device="cuda") if weights else None for n in "qk"}
    ws = None
    if weights:
        ws = torch.empty(ffi.qk_norm_rotate_workspace(c.x["q"], c.x["k"]), dtype=torch.uint8,
                         device="cuda")
    ffi.op_qk_norm_rotate_bwd(c.x["q"], c.x["k"], d["q"], d["k"], dx["q"], dx["k"], dw["q"],
                              dw["k"], ws, **c.kw)
    return d, dx, dw


def check_backward(c, d, dx, dw):
    u = torch.finfo(c.dtype).eps / 2
    cs, sn = c.tables()
    m = c.inside()
    for n in "qk":
        un, r, w = c.norm(n)
        e, size = turn(d[n].double(), cs, -sn if sn is not None else None, c.rot, c.pairs)
        gm = e * w
        mean = (gm * un).mean(-1, keepdim=True)
        ref = r * (gm - un * mean)
        tol = u * ref.abs() + 64 * 2.0 ** -24 * r * (
            (size * w.abs()) + un.abs() * ((size * w.abs() * un.abs()).mean(-1, keepdim=True)))
        got = dx[n].double()
        assert ((got - ref).abs() <= tol)[m].all(), (n, (got - ref).abs()[m].max().item())
        assert (got[~m] == FILL).all()
        if dw[n] is not None:
            terms = (e * un)[m].reshape(-1, c.dim)
            sizes = (size * un.abs())[m].reshape(-1, c.dim).sum(0)
            chain = terms.shape[0] / 64 + 64
            assert ((dw[n].double() - terms.sum(0)).abs() <= chain * 2.0 ** -24 * sizes).all()


@pytest.mark.parametrize("args", CASES, ids=str)
def test_backward(args):
    c = Case(*args[:7], pairs=args[7], layout=args[8])
    check_backward(c, *backward(c))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_tokens_and_heads(dtype):
    """More units than the backward's workgroups take in one round."""
    c = Case(dtype, 3, 1500, 16, 4, 64, 64)
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    c.check_forward(out)
    check_backward(c, *backward(c))


@pytest.mark.parametrize("lens", [[0, 5, 11], [11, 0, 1], [-3, 40, 7], [0, 0, 0]])
def test_padded_batches(lens):
    """What lies behind a sequence is neither read (NaN there) nor written nor counted."""
    c = Case(BF, 3, 11, 4, 2, 64, 32, lens=lens)
    pad = ~c.inside()
    for n in "qk":
        c.x[n][pad] = math.nan
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    c.check_forward(out)
    d, dx, dw = backward(c)
    check_backward(c, d, dx, dw)
    if not c.inside().any():
        assert (dw["q"] == 0).all() and (dw["k"] == 0).all()


def test_no_weights_no_positions_one_side():
    c = Case(BF, 2, 13, 4, 4, 64, 64, gamma=False, positions=False)
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    c.check_forward(out)
    d, dx, dw = backward(c, weights=False)
    check_backward(c, d, dx, dw)
    alone = c.empty("k")
    ffi.op_qk_norm_rotate(None, c.x["k"], None, alone, **c.kw)
    assert torch.equal(alone, out["k"])
    alone = c.empty("q")
    ffi.op_qk_norm_rotate(c.x["q"], None, alone, None, **c.kw)
    assert torch.equal(alone, out["q"])


def test_zero_tokens_give_zero_weight_gradients():
    c = Case(F32, 2, 0, 2, 2, 64, 64)
    _, _, dw = backward(c)
    assert (dw["q"] == 0).all() and (dw["k"] == 0).all()


def test_in_place_and_on_another_stream():
    c = Case(BF, 2, 50, 6, 6, 64, 64, layout="packed")
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], c.x["q"], c.x["k"], **c.kw)
    side.synchronize()
    for n in "qk":
        assert torch.equal(c.x[n].contiguous(), out[n])


def test_gradient_over_its_own_buffer():
    c = Case(BF, 2, 50, 6, 2, 128, 64)
    d, dx, dw = backward(c)
    ffi.op_qk_norm_rotate_bwd(c.x["q"], c.x["k"], d["q"], d["k"], d["q"], d["k"], **c.kw)
    for n in "qk":
        assert torch.equal(d[n], dx[n])


def test_position_outside_the_tables_is_nan_and_only_there():
    c = Case(F32, 1, 6, 2, 2, 64, 32)
    c.positions[0, 2], c.positions[0, 4] = -1, c.cos.shape[0]
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    for n in "qk":
        bad = torch.isnan(out[n][0]).all(1)                      # [tokens, dim], every head
        want = torch.zeros_like(bad)
        want[[2, 4], :32] = True
        assert torch.equal(bad, want) and not torch.isnan(out[n][0, :, :, 32:]).any()


def test_zeros_large_and_tiny_values():
    """A zero vector stays zero; 1e18 (squares near the top of fp32) and 1e-18 keep their
    direction."""
    c = Case(F32, 1, 4, 1, 1, 64, 0, gamma=False)
    c.x["q"][0, 0] = 0
    c.x["q"][0, 1] *= 1e17
    c.x["q"][0, 2] *= 1e-18
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    c.check_forward(out)
    assert (out["q"][0, 0] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("name", ["cos", "sin", "q_gamma", "k_gamma"])
def test_tables_at_any_address(dtype, pairs, name):
    """A table that starts 4 bytes behind a 16-byte boundary gives the same bits."""
    c = Case(dtype, 2, 21, 3, 2, 96, 80, pairs=pairs)
    want = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], want["q"], want["k"], **c.kw)
    d, dx, dw = backward(c)
    moved = torch.empty(c.kw[name].numel() + 1, device="cuda")[1:].view(c.kw[name].shape)
    assert moved.data_ptr() % 16 == 4
    moved.copy_(c.kw[name])
    c.kw[name] = moved
    out = {n: c.empty(n) for n in "qk"}
    ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
    _, dx2, dw2 = backward(c)
    for n in "qk":
        assert torch.equal(out[n], want[n])
        assert torch.equal(dx[n], dx2[n]) and torch.equal(dw[n], dw2[n])


def test_gradient_against_differences():
    c = Case(F32, 1, 3, 2, 1, 32, 32, seed=3)
    d, dx, dw = backward(c)

    def loss():
        out = {n: c.empty(n) for n in "qk"}
        ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
        return sum((out[n].double() * d[n].double()).sum().item() for n in "qk")

    # Central differences of step h: truncation ~ h^2, rounding ~ 2^-24 sqrt(n) / h.
    h = 2.0 ** -7
    for n, at in (("q", (0, 1, 0, 5)), ("q", (0, 2, 1, 31)), ("k", (0, 0, 0, 16))):
        x0 = c.x[n][at].item()
        f = []
        for step in (h, -h):
            c.x[n][at] = x0 + step
            f.append(loss())
        c.x[n][at] = x0
        assert abs((f[0] - f[1]) / (2 * h) - dx[n][at].item()) < 2e-3
    for n, i in (("q", 7), ("k", 20)):
        w0 = c.gamma[n][i].item()
        f = []
        for step in (h, -h):
            c.gamma[n][i] = w0 + step
            f.append(loss())
        c.gamma[n][i] = w0
        assert abs((f[0] - f[1]) / (2 * h) - dw[n][i].item()) < 2e-3


def test_captured_and_replayed():
    c = Case(BF, 2, 64, 8, 4, 64, 64)
    out = {n: c.empty(n) for n in "qk"}
    g = torch.Generator().manual_seed(1)
    d = {n: torch.randn(out[n].shape, generator=g).to(BF).cuda() for n in "qk"}
    dx = {n: c.empty(n) for n in "qk"}
    dw = {n: torch.zeros(c.dim, device="cuda") for n in "qk"}
    ws = torch.empty(ffi.qk_norm_rotate_workspace(c.x["q"], c.x["k"]), dtype=torch.uint8,
                     device="cuda")

    def both():
        ffi.op_qk_norm_rotate(c.x["q"], c.x["k"], out["q"], out["k"], **c.kw)
        ffi.op_qk_norm_rotate_bwd(c.x["q"], c.x["k"], d["q"], d["k"], dx["q"], dx["k"], dw["q"],
                                  dw["k"], ws, **c.kw)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        for n in "qk":
            c.x[n].copy_(torch.randn(c.x[n].shape, generator=g).to(BF))
        both()
        torch.cuda.synchronize()
        want = [t.clone() for n in "qk" for t in (out[n], dx[n], dw[n])]
        for n in "qk":
            for t in (out[n], dx[n], dw[n]):
                t.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        got = [t for n in "qk" for t in (out[n], dx[n], dw[n])]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
