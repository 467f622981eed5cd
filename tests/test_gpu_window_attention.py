"""Attention in a sliding window with sinks, forward and backward, against the
formulas in 64 bits.

Tolerances, element by element, with u = finfo(type).eps / 2 (one rounding to
the type) and e = 2^-24 (one of fp32).  A score is a sum of dim products: its
error is at most (dim + 4) e scale sum |q k|; the exponential's argument in base
2 adds 4 e of its size.  Call the largest such error of the row d; every weight
is then within f = 2 d + (n + 64) e of itself, relative (n keys are summed).
* o = sum p v: (u [p is rounded] + f) sum p |v| + u |o|; lse: d + 64 e (1 + |lse|)
  (fp32: no rounding of p, u = e).
* dv = sum p do: (u + f) sum p |do| + u |dv|.
* dS = p (dP - D): D comes from o, which is rounded: its error is u sum |do o|,
  that of dP is (dim + 4) e sum |do v|; so dS is within
  (f + u) |dS| + p (u sum |do o| + (dim + 4) e (sum |do v| + sum |do o|)), and dq
  and dk sum that against |k| and |q|, plus (n e + u) of the result's own sums.
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


def tensor(g, b, t, h, d, dtype, layout):
    if layout == "heads":                     # [b][head][t + 3][d]
        x = torch.randn(b, h, t + 3, d, generator=g).to(dtype).cuda()
        return x.transpose(1, 2)[:, 1:1 + t]
    if layout == "packed":                    # a third of [b][t][head][3][d]
        return torch.randn(b, t, h, 3, d, generator=g).to(dtype).cuda()[:, :, :, 1]
    return torch.randn(b, t, h, d, generator=g).to(dtype).cuda()


class Case:
    def __init__(self, dtype=BF, b=2, tq=70, tk=None, h=4, kv=2, d=64, causal=True, window=30,
                 sinks=3, q_lens=None, k_lens=None, layout="plain", scale=None, gain=1.5, seed=0):
        tk = tq if tk is None else tk
        g = torch.Generator().manual_seed(seed * 7919 + tq + 3 * tk + d)
        self.dtype, self.b, self.tq, self.tk, self.h, self.kv, self.d = dtype, b, tq, tk, h, kv, d
        self.causal, self.window, self.sinks = causal, window, sinks
        self.scale = 1 / math.sqrt(d) if scale is None else scale
        self.q = tensor(g, b, tq, h, d, dtype, layout)
        self.q.mul_(gain)
        self.k, self.v = (tensor(g, b, tk, kv, d, dtype, layout) for _ in range(2))
        self.dout = tensor(g, b, tq, h, d, dtype, layout)
        self.ql, self.kl = q_lens or [tq] * b, k_lens or [tk] * b
        self.q_lens = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32).cuda()
        self.k_lens = None if k_lens is None else torch.tensor(k_lens, dtype=torch.int32).cuda()
        self.ql = [min(max(n, 0), tq) for n in self.ql]
        self.kl = [min(max(n, 0), tk) for n in self.kl]
        self.kw = dict(sinks=sinks, causal=causal, scale=self.scale, q_lens=self.q_lens,
                       k_lens=self.k_lens)

    def workspace(self, backward=False):
        n = ffi.window_attention_workspace(self.q, self.k, self.window, self.sinks, self.causal,
                                           backward)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN where read unwritten

    def like(self, x):
        return torch.full(tuple(x.shape), FILL, dtype=x.dtype, device="cuda")

    def forward(self, lse=True, ws=None):
        o = self.like(self.q)
        l = torch.full((self.b, self.h, self.tq), FILL, device="cuda") if lse else None
        ffi.op_window_attention(self.q, self.k, self.v, o, self.window, lse=l,
                                workspace=self.workspace() if ws is None else ws, **self.kw)
        return o, l

    def backward(self, o, lse, ws=None):
        dq, dk, dv = (self.like(x) for x in (self.q, self.k, self.v))
        ffi.op_window_attention_bwd(self.q, self.k, self.v, o, lse, self.dout, dq, dk, dv,
                                    self.window, workspace=self.workspace(True) if ws is None else ws,
                                    **self.kw)
        return dq, dk, dv

    def mask(self, b):
        ql, kl = self.ql[b], self.kl[b]
        p = (torch.arange(ql) + kl - ql)[:, None]
        j = torch.arange(kl)[None]
        m = ((p - j).abs() < self.window) | (j < self.sinks)
        return m & (j <= p) if self.causal else m

    def heads(self):
        """Sequence and query head in 64 bits on the CPU: q, k, v, dout, mask, scores, weights."""
        q, k, v, do = (x.double().cpu() for x in (self.q, self.k, self.v, self.dout))
        grp = self.h // self.kv
        for b in range(self.b):
            m, ql, kl = self.mask(b), self.ql[b], self.kl[b]
            for h in range(self.h):
                qh, dh = q[b, :ql, h], do[b, :ql, h]
                kh, vh = k[b, :kl, h // grp], v[b, :kl, h // grp]
                s = (qh @ kh.T * self.scale).masked_fill(~m, -math.inf)
                lse = torch.logsumexp(s, 1) if kl else torch.full((ql,), -math.inf, dtype=s.dtype)
                p = torch.where(m, torch.exp(s - lse[:, None]), 0.0)
                size = torch.where(m, (qh.abs() @ kh.abs().T) * self.scale, 0.0)
                d = size.amax(1) if kl else torch.zeros(ql, dtype=s.dtype)
                d = ((self.d + 4) * E * d + 4 * E * (1 + d))[:, None]
                f = 2 * d + (kl + 64) * E
                yield b, h, qh, kh, vh, dh, m, lse, p, d[:, 0], f

    def exact_forward(self):
        """o and lse rounded to their types, for the backward pass's tests."""
        o = torch.zeros(self.b, self.tq, self.h, self.d, dtype=torch.float64)
        lse = torch.zeros(self.b, self.h, self.tq)
        for b, h, _, _, vh, _, _, l, p, _, _ in self.heads():
            o[b, :self.ql[b], h] = p @ vh
            lse[b, h, :self.ql[b]] = l.float()
        return o.to(self.dtype).cuda(), lse.cuda()

    def check_forward(self, o, lse):
        u = torch.finfo(self.dtype).eps / 2
        o = o.double().cpu()
        lse = None if lse is None else lse.double().cpu()
        for b, h, _, _, vh, _, m, l, p, d, f in self.heads():
            n = self.ql[b]
            ref = p @ vh
            tol = ((u if self.dtype == BF else 0) + f) * (p @ vh.abs()) + u * ref.abs()
            err = (o[b, :n, h] - ref).abs()
            assert (err <= tol).all(), (b, h, err.max().item(), tol.max().item())
            assert (o[b, n:, h] == FILL).all(), "rows behind a sequence were written"
            if lse is None:
                continue
            some = m.any(1) if m.numel() else torch.zeros(n, dtype=torch.bool)
            assert (lse[b, h, :n][~some] == -math.inf).all()
            assert (o[b, :n, h][~some] == 0).all()
            e = (lse[b, h, :n] - l).abs()[some]
            assert (e <= (d + 64 * E * (1 + l.abs()))[some]).all()
            assert (lse[b, h, n:] == FILL).all()

    def check_backward(self, o, dq, dk, dv):
        u = torch.finfo(self.dtype).eps / 2
        ur = u if self.dtype == BF else 0.0               # rounding of P and dS as operands
        o = o.double().cpu()
        got = [x.double().cpu() for x in (dq, dk, dv)]
        ref = [torch.zeros(tuple(x.shape), dtype=torch.float64) for x in (dq, dk, dv)]
        tol = [torch.zeros_like(x) for x in ref]
        grp = self.h // self.kv
        for b, h, qh, kh, vh, dh, m, l, p, d, f in self.heads():
            ql, kl = self.ql[b], self.kl[b]
            oh = o[b, :ql, h]
            dp = dh @ vh.T
            D = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - D)
            sizes = (dh * oh).abs().sum(1, keepdim=True)
            # lse is rounded to fp32 on its way in.
            f = f + 8 * E * (1 + torch.where(l > -math.inf, l.abs(), 0.0))[:, None]
            dds = (f + ur) * ds.abs() + p * (u * sizes + (self.d + 4) * E * (dh.abs() @ vh.abs().T + sizes))
            n = (max(ql, kl) * grp + 64) * E
            ref[0][b, :ql, h] = ds @ kh * self.scale
            tol[0][b, :ql, h] = (dds + n * ds.abs()) @ kh.abs() * self.scale
            ref[1][b, :kl, h // grp] += ds.T @ qh * self.scale
            tol[1][b, :kl, h // grp] += (dds + n * ds.abs()).T @ qh.abs() * self.scale
            ref[2][b, :kl, h // grp] += p.T @ dh
            tol[2][b, :kl, h // grp] += ((f + ur + n) * p).T @ dh.abs()
        for i, name in enumerate(("dq", "dk", "dv")):
            lens = self.ql if name == "dq" else self.kl
            err = (got[i] - ref[i]).abs()
            ok = err <= tol[i] + u * ref[i].abs()
            for b in range(self.b):
                assert ok[b, :lens[b]].all(), (name, b, err[b, :lens[b]].max().item())
                assert (got[i][b, lens[b]:] == FILL).all(), name + ": written behind a sequence"


CASES = [
    dict(),
    dict(dtype=F32),
    dict(tq=1, tk=1, window=1, sinks=0),
    dict(tq=1, tk=1, dtype=F32, d=128, window=5, sinks=64),
    dict(tq=33, window=1, sinks=0, kv=4),                       # each token sees itself
    dict(tq=130, d=128, window=17, sinks=64, h=3, kv=1),
    dict(tq=129, d=128, window=64, sinks=1, dtype=F32, h=2, kv=1),
    dict(tq=200, causal=False, window=25, sinks=1, h=3, kv=3),
    dict(tq=197, causal=False, window=1 << 31, sinks=0, h=3, kv=3, layout="packed"),
    dict(tq=150, causal=False, window=40, sinks=20, dtype=F32, layout="packed", kv=4),
    dict(tq=300, window=64, sinks=4, layout="heads", h=8, kv=2, b=1),
    dict(tq=257, window=1000, sinks=0, b=1, h=5, kv=5),         # plain causal attention
    dict(tq=320, window=100, sinks=64, b=1, h=12, kv=1, d=128),
    dict(tq=6, tk=90, window=20, sinks=2),                      # a few new tokens on a cache
    dict(tq=6, tk=90, window=20, sinks=2, dtype=F32, d=128, layout="heads"),
    dict(tq=40, tk=100, causal=False, window=9, sinks=5, h=2, kv=1),
    dict(tq=100, tk=40, window=16, sinks=3),                    # the first 60 rows see nothing
    dict(tq=100, tk=40, causal=False, window=8, sinks=0, dtype=F32),
    dict(tq=90, b=4, q_lens=[90, 1, 0, 33], k_lens=[90, 1, 0, 33]),
    dict(tq=90, b=4, q_lens=[90, 1, 0, 33], k_lens=[64, 90, 31, 0], dtype=F32),
    dict(tq=70, b=3, q_lens=[70, -5, 200], k_lens=[3, 70, 500], causal=False, sinks=40, window=5),
    dict(tq=65, b=3, k_lens=[65, 0, 32], d=128, window=10),
    dict(tq=1100, b=1, h=2, kv=2, window=90, sinks=4),          # sinks' rows in several parts
    dict(tq=1300, b=1, h=2, kv=1, window=33, sinks=7, causal=False),
    dict(tq=700, b=1, h=8, kv=1, window=600, sinks=5, d=128),   # few key heads: rows in parts
    dict(tq=1500, b=1, h=4, kv=1, window=100, sinks=40, d=128, k_lens=[1400], dtype=F32),
    dict(tq=600, b=2, h=6, kv=1, causal=False, window=300, q_lens=[600, 77], k_lens=[500, 90]),
    dict(tq=1200, b=2, h=1, kv=1, window=50, sinks=64, dtype=F32, q_lens=[1200, 700],
         k_lens=[1200, 700]),
]


@pytest.mark.parametrize("kw", CASES, ids=str)
def test_forward(kw):
    c = Case(**kw)
    c.check_forward(*c.forward())


@pytest.mark.parametrize("kw", CASES, ids=str)
def test_backward(kw):
    c = Case(**kw)
    o, lse = c.exact_forward()
    c.check_backward(o, *c.backward(o, lse))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [700, 4000])
def test_single_tokens_on_long_caches(dtype, d, window):
    """Keys split over workgroups and joined; caches that end inside a tile, and empty ones."""
    c = Case(dtype=dtype, b=5, tq=1, tk=2500, h=8, kv=2, d=d, window=window, sinks=5,
             k_lens=[2500, 1, 0, 1023, 705], layout="heads")
    assert ffi.window_attention_workspace(c.q, c.k, window, 5) > 0
    c.check_forward(*c.forward())
    c.check_forward(c.forward(lse=False)[0], None)


def test_rows_split_over_keys():
    """More than 32 rows on few sequences: the tiles of a row block are split as well."""
    c = Case(b=1, tq=50, tk=3000, h=2, kv=1, window=5000, sinks=0)
    assert ffi.window_attention_workspace(c.q, c.k, 5000, 0) > 0
    c.check_forward(*c.forward())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_lies_behind_a_sequence_may_be_anything(dtype):
    c = Case(dtype=dtype, b=3, tq=100, q_lens=[100, 37, 0], k_lens=[100, 37, 0], window=50)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    for b in range(3):
        n = c.ql[b]
        for x in (c.q, c.k, c.v, c.dout, o):
            x[b, n:] = math.nan
        lse[b, :, n:] = math.nan
    o2, lse2 = c.forward()
    for b in range(3):
        assert torch.equal(o2[b, :c.ql[b]], o[b, :c.ql[b]])
    for a, b in zip(grads, c.backward(o, lse)):
        assert torch.equal(a, b)


def test_peaked_and_flat_scores():
    """Scores of hundreds (one key takes all) and of zero (all keys alike)."""
    for gain in (60.0, 0.0):
        for dtype in (BF, F32):
            c = Case(dtype=dtype, tq=150, window=70, gain=gain, seed=2)
            c.check_forward(*c.forward())


def test_large_window_equals_the_framework_attention():
    """An open window without sinks, both ways of asking for the same attention: each side's
    probabilities are rounded once (u) and its result once."""
    g = torch.Generator().manual_seed(3)
    b, t, h = 3, 197, 4
    qkv = torch.randn(b, t, h, 3, 64, generator=g).to(BF).cuda()
    o = torch.zeros(b, t, h, 64, dtype=BF, device="cuda")
    ffi.op_attention(ffi.BF16, qkv, 3 * h * 64, o, h * 64, b, t, h, 64, 0.125)
    o2 = torch.zeros_like(o)
    q, k, v = qkv[:, :, :, 0], qkv[:, :, :, 1], qkv[:, :, :, 2]
    ws = torch.empty(ffi.window_attention_workspace(q, k, t, causal=False), dtype=torch.uint8,
                     device="cuda")
    ffi.op_window_attention(q, k, v, o2, t, causal=False, workspace=ws)
    u = torch.finfo(BF).eps / 2
    big = v.abs().float().amax(1).double()[:, None]                # bounds sum p |v|
    assert ((o.double() - o2.double()).abs() <= 4 * u * big).all()


def test_gradients_against_differences():
    c = Case(dtype=F32, b=1, tq=40, h=2, kv=1, window=12, sinks=2, gain=0.7, seed=4)
    o, lse = c.forward()
    grads = dict(zip(("q", "k", "v"), c.backward(o, lse)))

    def loss():
        return (c.forward()[0].double() * c.dout.double()).sum().item()

    h = 2.0 ** -6                       # truncation ~ h^2, rounding ~ 2^-22 sqrt(2560) / h
    for n, at in (("q", (0, 20, 1, 3)), ("k", (0, 1, 0, 9)), ("k", (0, 30, 0, 60)),
                  ("v", (0, 0, 0, 5)), ("v", (0, 39, 0, 63))):
        x = getattr(c, n)
        x0 = x[at].item()
        f = []
        for step in (h, -h):
            x[at] = x0 + step
            f.append(loss())
        x[at] = x0
        assert abs((f[0] - f[1]) / (2 * h) - grads[n][at].item()) < 5e-3, (n, at)


def test_same_bits_every_time_and_on_another_stream():
    c = Case(b=2, tq=600, window=100, h=8, kv=2, d=128)
    o, lse = c.forward()
    g = c.backward(o, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = c.forward()
        g2 = c.backward(o2, lse2)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(a, b) for a, b in zip(g, g2))


def test_two_calls_at_once_with_a_workspace_each():
    cs = [Case(b=3, tq=1, tk=2000, h=8, kv=1, window=3000, seed=i) for i in range(2)]
    want = [c.forward() for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    ws = [c.workspace() for c in cs]
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for c, s, w in zip(cs, streams, ws):
            with torch.cuda.stream(s):
                outs.append(c.forward(ws=w))
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(outs):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])


def test_captured_and_replayed_with_growing_caches():
    """One graph of a decoding step: the lengths are read when it runs."""
    c = Case(b=3, tq=1, tk=1500, h=8, kv=2, window=600, sinks=4, k_lens=[100, 700, 1400])
    ws = c.workspace()
    o, lse = c.like(c.q), torch.zeros(c.b, c.h, 1, device="cuda")

    def step():
        ffi.op_window_attention(c.q, c.k, c.v, o, c.window, lse=lse, workspace=ws, **c.kw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        c.kl = [n + 20 for n in c.kl]
        c.k_lens.copy_(torch.tensor(c.kl, dtype=torch.int32))
        o.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        c.check_forward(o, lse)


def test_captured_training_step():
    c = Case(b=1, tq=1100, h=4, kv=2, window=90, sinks=4)
    o, lse = c.forward()
    ws, wb = c.workspace(), c.workspace(True)
    dq, dk, dv = (c.like(x) for x in (c.q, c.k, c.v))

    def step():
        ffi.op_window_attention(c.q, c.k, c.v, o, c.window, lse=lse, workspace=ws, **c.kw)
        ffi.op_window_attention_bwd(c.q, c.k, c.v, o, lse, c.dout, dq, dk, dv, c.window,
                                    workspace=wb, **c.kw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    gen = torch.Generator().manual_seed(9)
    for _ in range(3):
        c.q.copy_(torch.randn(c.q.shape, generator=gen).to(BF))
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (o, lse, dq, dk, dv)]
        for x in (o, dq, dk, dv):
            x.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, lse, dq, dk, dv), want))


def test_cache_offsets_beyond_four_gigabytes():
    """A cache whose last tokens lie past 2^32 bytes, 16 MiB from token to token."""
    tk, d = 300, 64
    stride = (1 << 24) // 2
    buf = torch.zeros(stride * (tk - 1) + d, dtype=BF, device="cuda")
    k = torch.as_strided(buf, (1, tk, 1, d), (buf.numel(), stride, d, 1))
    c = Case(b=1, tq=1, tk=tk, h=2, kv=1, window=1000, sinks=0)
    k.copy_(c.k)
    want, l1 = c.forward()
    o, lse = c.like(c.q), torch.zeros(1, 2, 1, device="cuda")
    ffi.op_window_attention(c.q, k, c.v, o, c.window, lse=lse, workspace=c.workspace(), **c.kw)
    assert torch.equal(o, want) and torch.equal(lse, l1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_heads_four_gigabytes_apart(dtype):
    """q, k, v and dout of each head in one place, the next head 2^32 bytes on: the same bits as
    side by side."""
    t, d = 150, 64
    c = Case(dtype=dtype, b=1, tq=t, h=2, kv=2, window=40, sinks=3)
    o, lse = c.forward()
    want = (o, lse, *c.backward(o, lse))
    far = (1 << 32) // c.q.element_size()
    buf = torch.zeros(far + 4 * t * d, dtype=dtype, device="cuda")
    for i, n in enumerate(("q", "k", "v", "dout")):
        x = torch.as_strided(buf, (1, t, 2, d), (2 * far, d, far, 1), i * t * d)
        x.copy_(getattr(c, n))
        setattr(c, n, x)
    o2, lse2 = c.forward()
    assert all(torch.equal(x, y) for x, y in zip(want, (o2, lse2, *c.backward(o2, lse2))))


def test_gradients_of_large_and_odd_groups():
    """Groups that do not divide a tile of rows, and one larger than it."""
    for h, kv, dtype in ((7, 1, BF), (33, 1, F32), (40, 1, BF), (71, 1, BF), (130, 2, F32)):
        c = Case(dtype=dtype, b=1, tq=37, h=h, kv=kv, window=11, sinks=2)
        o, lse = c.exact_forward()
        c.check_backward(o, *c.backward(o, lse))
        c.check_forward(*c.forward())


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("tq,tk,window,sinks,causal,k_lens", [
    (1, 700, 100, 4, True, [700, 333]),     # one new token: a window and sinks in a cache
    (1, 700, 64, 0, True, [700, 50]),
    (37, 900, 70, 40, True, [900, 411]),    # the window of the first query starts inside a tile
    (37, 900, 70, 33, False, [850, 200]),
    (5, 40, 3, 1, False, [40, 7]),
    (260, 1000, 130, 64, True, [1000, 300]),
])
def test_keys_that_no_query_sees(dtype, d, tq, tk, window, sinks, causal, k_lens):
    """NaN in keys and values that no query of the sequence sees changes no bit."""
    c = Case(dtype=dtype, tq=tq, tk=tk, h=6, kv=2, d=d, window=window, sinks=sinks, causal=causal,
             k_lens=k_lens, layout="heads")
    hidden = [torch.ones(tk, dtype=torch.bool) for _ in range(2)]
    for b in range(2):
        hidden[b][:c.kl[b]] = ~c.mask(b).any(0)
        assert hidden[b].any() and not hidden[b].all()
    results = []
    for value in (0.0, math.nan, math.inf):
        for b in range(2):
            at = torch.nonzero(hidden[b])[:, 0].cuda()
            c.k[b, at], c.v[b, at] = value, value
        o, lse = c.forward()
        results.append((o, lse, *c.backward(o, lse)))
    for got in results[1:]:
        for x, y in zip(results[0], got):
            assert torch.equal(x, y)
    assert all(bool(torch.isfinite(x).all()) for x in results[0])
    for b in range(2):
        at = torch.nonzero(hidden[b][:c.kl[b]])[:, 0].cuda()
        assert not results[0][3][b, at].any() and not results[0][4][b, at].any()
