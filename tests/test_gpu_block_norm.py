"""The step between two blocks (norm, gate, residual addition, norm), forward and
backward, against the formulas in 64 bits.

Tolerances, with h = 2^-24 (half a step of fp32) and chains of at most c = dim / 64 + 32
roundings (a lane sums dim / 64 values or fewer, lanes and waves add 10).  A normed value
v^ = (v - mean) r: the mean is off by c h mean|v|, the difference by h of its parts, and r
relatively by rho = c h (1 + A r), A = max|v| + mean|v|: |error| <= hat = c h A r (1 + |v^|) +
rho |v^|.  An error e of v itself adds r (e + mean e) + |v^| r rms(e).  Through a norm, with d the
gradient times gamma: |error| <= r (c h (|d| + |v^| mean|d v^| + mean|d|) + hat |mean(d v^)| + |v^|
mean(|d| hat)) + rho |result|, and an error e of d adds r (e + |v^| mean(e |v^|) + mean e).
A product and a sum: 3 h of the parts.  Results are rounded once, by u = finfo(type).eps / 2; sums
over n tokens: (n + 64) h of the sum of the sizes, and the terms' own errors.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10018_amd import ffi  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FILL = 7.0
H = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


def mean(v):
    return v.mean(-1, keepdim=True)


class Normed:
    """v normalised, with what the tolerances need; e: how far v itself may be off."""

    def __init__(self, v, eps, layer, e=None):
        self.c = (v.shape[-1] / 64 + 32) * H
        mu = mean(v) if layer else torch.zeros_like(v[..., :1])
        self.r = 1 / torch.sqrt(mean((v - mu) ** 2) + eps)
        self.v = (v - mu) * self.r
        a = v.abs().amax(-1, keepdim=True) + mean(v.abs())
        self.rho = self.c * (1 + a * self.r)
        self.hat = self.c * a * self.r * (1 + self.v.abs()) + self.rho * self.v.abs()
        if e is not None:
            self.hat = self.hat + self.r * (e + mean(e)) + self.v.abs() * self.r * mean(e * e).sqrt()
            self.rho = self.rho + self.r * mean(e * e).sqrt()
        self.layer = layer

    def affine(self, gamma, beta):
        out = self.v * gamma + beta
        return out, self.hat * gamma.abs() + 3 * H * ((self.v * gamma).abs() + beta.abs())

    def back(self, d, e):
        """The gradient through the norm, and its tolerance; d times gamma, off by e."""
        m1, m2 = mean(d * self.v), mean(d) if self.layer else 0.0
        out = self.r * (d - self.v * m1 - m2)
        va, da = self.v.abs(), d.abs()
        tol = self.r * (self.c * (da + va * mean(da * va) + mean(da)) + self.hat * m1.abs() + va * mean(da * self.hat))
        tol = tol + self.rho * out.abs() + self.r * (e + va * mean(e * va) + mean(e))
        return out, tol


class Case:
    def __init__(self, dtype, stream, b, t, d, kind="rms", post=True, gate="shared", affine=True, lens=None,
                 strided=False, seed=0, offset=0, scale=0.9, shift=0.0):
        g = torch.Generator().manual_seed(seed + b + t + d)
        self.dtype, self.stream, self.b, self.t, self.d = dtype, stream, b, t, d
        self.layer, self.post, self.strided, self.offset = kind == "layer", post, strided, offset
        self.x = self.place(torch.randn(b, t, d, generator=g) * 1.5 + shift, stream)
        self.y = self.place(torch.randn(b, t, d, generator=g) * 0.8 - shift, dtype)
        self.dx_out = self.place(torch.randn(b, t, d, generator=g), stream)
        self.du = self.place(torch.randn(b, t, d, generator=g), dtype)
        vec = lambda on, mid, shape=(d,): (mid + 0.3 * torch.randn(shape, generator=g)).cuda() if on else None  # noqa: E731
        self.w = dict(pre_gamma=vec(affine, 1), pre_beta=vec(affine and self.layer, 0),
                      post_gamma=vec(affine and post, 1), post_beta=vec(affine and post and self.layer, 0),
                      gate={"none": None, "shared": vec(True, 0.5), "sequence": vec(True, 0.5, (b, d))}[gate])
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
        self.eps, self.scale = 1e-5, scale
        self.kw = dict(post_norm=post, lens=self.lens, residual_scale=scale, eps=self.eps, kind=kind, **self.w)

    def place(self, v, dtype):
        """v on the device; strided: [tokens][batch][dim + 5] with an offset (no 16-byte steps)."""
        v = v.to(dtype)
        if not self.strided:
            return v.cuda()
        buf = torch.full((self.t, self.b, self.d + 5 + self.offset), FILL, dtype=dtype, device="cuda")
        out = buf[:, :, 1 + self.offset:1 + self.offset + self.d].transpose(0, 1)
        out.copy_(v)
        return out

    def empty(self, dtype):
        return self.place(torch.full((self.b, self.t, self.d), FILL), dtype)

    def inside(self):
        m = torch.ones(self.b, self.t, dtype=torch.bool, device="cuda")
        if self.lens is not None:
            m = torch.arange(self.t, device="cuda")[None] < self.lens[:, None]
        return m

    def weight(self, n, none):
        w = self.w[n]
        if w is None:
            return torch.full((self.d,), none, dtype=torch.float64, device="cuda")
        return w.double()[:, None] if w.dim() == 2 else w.double()

    def branch(self, y):
        """n, its tolerance, and the norm (or None)."""
        if not self.post:
            return y, torch.zeros_like(y), None
        n = Normed(y, self.eps, self.layer)
        return *n.affine(self.weight("post_gamma", 1.0), self.weight("post_beta", 0.0)), n

    def forward(self):
        out = self.empty(self.stream), self.empty(self.dtype)
        ffi.op_block_norm(self.x, self.y, *out, **self.kw)
        return out

    def check_forward(self, x_out, u, with_y=True):
        m = self.inside()
        x = torch.where(m[..., None], self.x.double(), 1.0)
        ref, e = self.scale * x, H * (self.scale * x).abs()
        if with_y:
            n, tn, _ = self.branch(torch.where(m[..., None], self.y.double(), 1.0))
            g = self.weight("gate", 1.0)
            e = g.abs() * tn + 3 * H * (ref.abs() + (g * n).abs())
            ref = ref + g * n
        if x_out is not None:
            tol = e + torch.finfo(self.stream).eps / 2 * ref.abs()
            self.holds("x_out", x_out, ref, tol, m)
        if u is not None:
            v, tol = Normed(ref, self.eps, self.layer, e).affine(self.weight("pre_gamma", 1.0), self.weight("pre_beta", 0.0))
            self.holds("u", u, v, tol + torch.finfo(self.dtype).eps / 2 * v.abs(), m)

    def holds(self, name, got, ref, tol, m):
        bad = ~((got.double() - ref).abs() <= tol + 1e-37)[m]
        assert not bad.any(), (name, int(bad.sum()), ((got.double() - ref).abs() / tol)[m].max())
        assert (got[~m] == FILL).all(), "rows behind a sequence were written"
        if self.strided:  # between a row's end and the next one's start
            gap, n = 5 + self.offset, self.t * self.b - 1
            around = torch.as_strided(got, (n, gap), (self.d + gap, 1), got.storage_offset() + self.d)
            assert (around == FILL).all(), "written beside the rows"

    def backward(self, dx_out=True, du=True, y=True, weights=True):
        names = [n for n in self.w if self.w[n] is not None and weights and (du or not n.startswith("pre"))]
        out = {"d_" + n: torch.full_like(self.w[n], math.nan) for n in names}
        ws = torch.full((ffi.block_norm_workspace(self.y, self.w["gate"]),), 0xff, dtype=torch.uint8, device="cuda")
        dx, dy = self.empty(self.stream), self.empty(self.dtype) if y else None
        ffi.op_block_norm_bwd(self.x if du else None, self.y if y else None, self.dx_out if dx_out else None,
                              self.du if du else None, dx, dy, workspace=ws, **self.kw, **out)
        return dict(dx=dx, dy=dy, **out)

    def check_backward(self, got, dx_out=True, du=True, y=True):
        """self.x stands for the forward's x_out."""
        m = self.inside()
        keep = lambda v: torch.where(m[..., None], v.double(), 0.0)  # noqa: E731
        x = torch.where(m[..., None], self.x.double(), 1.0)
        n = int(m.sum())
        chain = (n + 64) * H
        sums = {}
        d = torch.zeros_like(x)
        e = torch.zeros_like(x)
        if du:
            nx = Normed(x, self.eps, self.layer)
            dul = keep(self.du)
            g = self.weight("pre_gamma", 1.0)
            sums["d_pre_gamma"] = dul * nx.v, dul.abs() * nx.hat
            sums["d_pre_beta"] = dul, torch.zeros_like(dul)
            d, e = nx.back(dul * g, H * (dul * g).abs())
        if dx_out:
            e = e + 2 * H * (keep(self.dx_out).abs() + d.abs())
            d = d + keep(self.dx_out)
        tol = abs(self.scale) * (e + 2 * H * d.abs())
        self.holds("dx", got["dx"], self.scale * d, tol + torch.finfo(self.stream).eps / 2 * (self.scale * d).abs(), m)
        if y:
            v, tv, ny = self.branch(torch.where(m[..., None], self.y.double(), 1.0))
            sums["d_gate"] = d * v, e * v.abs() + d.abs() * tv
            g = self.weight("gate", 1.0)
            dn, e = d * g, e * g.abs() + H * (d * g).abs()
            if self.post:
                sums["d_post_gamma"] = dn * ny.v, e * ny.v.abs() + dn.abs() * ny.hat
                sums["d_post_beta"] = dn, e
                pg = self.weight("post_gamma", 1.0)
                dn, e = ny.back(dn * pg, e * pg.abs() + H * (dn * pg).abs())
            self.holds("dy", got["dy"], dn, e + torch.finfo(self.dtype).eps / 2 * dn.abs(), m)
        for name, (term, err) in sums.items():
            if got.get(name) is None:
                continue
            over = (1,) if name == "d_gate" and self.w["gate"].dim() == 2 else (0, 1)
            tol = (err + chain * term.abs()).sum(over)
            off = (got[name].double() - term.sum(over)).abs()
            assert (off <= tol + 1e-37).all(), (name, (off / tol).max())


DIMS = [1, 2, 7, 8, 64, 65, 512, 520, 768, 1000, 1025, 2048, 2050, 4096, 4104, 8192, 8200, 12001, 16384]
TYPES = [(BF, BF), (BF, F32), (F32, F32)]


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("d", DIMS)
def test_widths(dtype, stream, d):
    """Every width's kernels, both norms, rows that do not fill a workgroup."""
    for kind in ("rms", "layer"):
        c = Case(dtype, stream, 2, 7, d, kind=kind, gate="sequence")
        c.check_forward(*c.forward())
        c.check_backward(c.backward())


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", ["none", "shared", "sequence"])
@pytest.mark.parametrize("affine", [True, False])
def test_forms(dtype, stream, kind, post, gate, affine):
    c = Case(dtype, stream, 3, 50, 192, kind=kind, post=post, gate=gate, affine=affine)
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("b,t,d", [(1, 1, 768), (5, 1, 40), (1, 3000, 96), (1500, 2, 24), (2000, 1, 16), (3, 700, 2056)])
def test_batches(dtype, stream, b, t, d):
    """Many tokens of one sequence, many sequences of one token, gates of either kind."""
    for gate in ("shared", "sequence"):
        c = Case(dtype, stream, b, t, d, gate=gate)
        c.check_forward(*c.forward())
        c.check_backward(c.backward())


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("d", [24, 513, 2048, 5000])
def test_strides(dtype, stream, d):
    for offset in (0, 2):
        c = Case(dtype, stream, 3, 5, d, kind="layer", strided=True, offset=offset)
        c.check_forward(*c.forward())
        c.check_backward(c.backward())


@pytest.mark.parametrize("d", [72, 1500, 2500])
@pytest.mark.parametrize("lens", [[0, 5, 11], [11, 0, 1], [-3, 40, 7], [0, 0, 0]])
def test_padded_batches(d, lens):
    """What lies behind a sequence is neither read (NaN there) nor written nor counted."""
    for gate in ("shared", "sequence"):
        c = Case(BF, F32, 3, 11, d, kind="layer", gate=gate, lens=lens)
        pad = ~c.inside()
        for v in (c.x, c.y, c.dx_out, c.du):
            v[pad] = math.nan
        c.check_forward(*c.forward())
        c.check_backward(c.backward())


@pytest.mark.parametrize("dtype,stream", TYPES)
def test_parts_left_out(dtype, stream):
    c = Case(dtype, stream, 2, 20, 320, kind="layer")
    x_out, u = c.forward()
    for got in ((c.empty(stream), None), (None, c.empty(dtype))):
        ffi.op_block_norm(c.x, c.y, *got, **c.kw)
        assert all(g is None or torch.equal(g, full) for g, full in zip(got, (x_out, u)))
    c.check_backward(c.backward(dx_out=False), dx_out=False)
    c.check_backward(c.backward(du=False), du=False)
    full, bare = c.backward(), c.backward(weights=False)
    assert torch.equal(full["dx"], bare["dx"]) and torch.equal(full["dy"], bare["dy"])
    # No block output: the norm ahead of the first block.
    c = Case(dtype, stream, 2, 20, 320, post=False, gate="none", scale=1.0)
    out = c.empty(stream), c.empty(dtype)
    ffi.op_block_norm(c.x, None, *out, **c.kw)
    c.check_forward(*out, with_y=False)
    c.check_backward(c.backward(y=False), y=False)


@pytest.mark.parametrize("dtype,stream", [(BF, BF), (F32, F32)])
def test_in_place(dtype, stream):
    c = Case(dtype, stream, 2, 30, 768)
    x_out, u = c.forward()
    x, y = c.x.clone(), c.y.clone()
    ffi.op_block_norm(x, y, x, y, **c.kw)
    assert torch.equal(x, x_out) and torch.equal(y, u)
    ref = c.backward()
    for dx_is, dy_is in ((0, 1), (2, 3)):
        t = [v.clone() for v in (c.dx_out, c.du, c.x, c.y)]
        ffi.op_block_norm_bwd(t[2], t[3], t[0], t[1], t[dx_is], t[dy_is], **c.kw)
        assert torch.equal(t[dx_is], ref["dx"]) and torch.equal(t[dy_is], ref["dy"])


def test_far_means_keep_their_digits():
    """A mean of 4096 against a spread of 1: the tolerances' A r is some thousands, no more."""
    c = Case(F32, F32, 2, 9, 1000, kind="layer", shift=4096.0)
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


def test_zeros_and_large_values():
    c = Case(F32, F32, 1, 4, 200, post=True, gate="none")
    c.x[0, 0], c.y[0, 0] = 0.0, 0.0
    c.x[0, 1] *= 1e15
    c.y[0, 2] *= 1e-15
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


def test_a_spoiled_token_spoils_itself_alone():
    c = Case(BF, F32, 2, 9, 768, kind="layer")
    x_out, u = c.forward()
    c.x[0, 3, 5], c.y[1, 7, 700] = math.nan, math.inf
    x2, u2 = c.forward()
    m = torch.ones(2, 9, dtype=torch.bool)
    m[0, 3] = m[1, 7] = False
    assert torch.equal(x_out[m], x2[m]) and torch.equal(u[m], u2[m])
    assert u2[0, 3].isnan().all() and u2[1, 7].isnan().all()


def test_no_tokens():
    for b, t in ((0, 5), (3, 0)):
        for gate in ("shared", "sequence"):
            c = Case(BF, BF, b, t, 40, kind="layer", gate=gate)
            c.forward()
            got = c.backward()
            assert all((got[n] == 0).all() for n in got if n.startswith("d_"))


def test_gradients_against_differences():
    """The weighted sum of the results moves as the gradients say when x, y and every weight move by t D
    to either side.  In 64 bits on the CPU the sum's third derivative along D is estimated from steps four
    times as wide (its share of the difference falls with t^2), doubled; the fp32 sums' own errors are their
    tolerances over t."""
    c = Case(F32, F32, 2, 6, 48, kind="layer", gate="sequence", scale=0.8)
    g = torch.Generator().manual_seed(1)
    par = {n: v for n, v in c.w.items()}
    par.update(x=c.x, y=c.y)
    step = {n: torch.randn(v.shape, generator=g).cuda() for n, v in par.items()}
    before = {n: v.clone() for n, v in par.items()}

    def total(t):
        v = {n: (before[n] + t * step[n]).double() for n in par}
        norm = lambda z, a: ((z - mean(z)) / torch.sqrt(mean((z - mean(z)) ** 2) + c.eps) * v[a + "_gamma"]  # noqa: E731
                             + v[a + "_beta"])
        x = c.scale * v["x"] + v["gate"][:, None] * norm(v["y"], "post")
        return (x * c.dx_out.double()).sum() + (norm(x, "pre") * c.du.double()).sum()

    x_out, _ = c.forward()
    c.x = x_out                      # what the backward pass is given
    got = c.backward()
    said = sum((got[("d" if n in "xy" else "d_") + n].double() * step[n].double()).sum() for n in par)
    t = 2.0 ** -8
    near, far = ((total(s) - total(-s)) / (2 * s) for s in (t, 4 * t))
    # far - near is 15 t^2 / 6 of the third derivative, near off by t^2 / 6 of it.
    size = sum((got[("d" if n in "xy" else "d_") + n].abs().double() * step[n].abs().double()).sum() for n in par)
    assert abs(near - said) <= 2 * abs(far - near) / 15 + 2048 * H * size


def test_same_bits_every_time_and_on_another_stream():
    c = Case(BF, F32, 3, 400, 768, gate="sequence")
    first = c.backward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        second = c.backward()
    s.synchronize()
    assert all(torch.equal(first[n], second[n]) for n in first)


def test_captured_and_replayed():
    c = Case(BF, BF, 2, 60, 768, kind="layer")
    x_out, u, dx, dy = c.empty(BF), c.empty(BF), c.empty(BF), c.empty(BF)
    out = {"d_" + n: torch.empty_like(v) for n, v in c.w.items()}
    ws = torch.empty(ffi.block_norm_workspace(c.y, c.w["gate"]), dtype=torch.uint8, device="cuda")

    def step():
        ffi.op_block_norm(c.x, c.y, x_out, u, **c.kw)
        ffi.op_block_norm_bwd(x_out, c.y, c.dx_out, c.du, dx, dy, workspace=ws, **c.kw, **out)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for i in range(4):
        c.y.copy_(torch.randn(c.y.shape, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (x_out, u, dx, dy, *out.values())]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (x_out, u, dx, dy, *out.values())))


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("d", [3, 100, 128, 129, 200, 256, 257, 4097, 8191, 8193, 12002])
def test_rows_that_share_a_wave_and_rows_of_columns_apart(dtype, stream, d):
    """Rows of 16 and of 32 lanes, ends of rows inside a run, rows whose weights' sums are taken apart:
    padded batches, unaligned rows, gates of either kind."""
    for kind, gate, strided in (("rms", "shared", True), ("layer", "sequence", False), ("layer", "shared", True)):
        c = Case(dtype, stream, 3, 37, d, kind=kind, gate=gate, lens=[37, 0, 19], strided=strided, offset=1)
        pad = ~c.inside()
        for v in (c.x, c.y, c.dx_out, c.du):
            v[pad] = math.nan
        c.check_forward(*c.forward())
        c.check_backward(c.backward())
        c.check_backward(c.backward(dx_out=False), dx_out=False)
        c.check_backward(c.backward(du=False), du=False)


@pytest.mark.parametrize("dtype,stream", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("d", [90, 250, 6001, 9000])
def test_in_place_with_the_weights_gradients(dtype, stream, d):
    c = Case(dtype, stream, 2, 30, d, kind="layer", gate="sequence")
    x_out, u = c.forward()
    x, y = c.x.clone(), c.y.clone()
    ffi.op_block_norm(x, y, x, y, **c.kw)
    assert torch.equal(x, x_out) and torch.equal(y, u)
    ref = c.backward()
    ws = torch.empty(ffi.block_norm_workspace(c.y, c.w["gate"]), dtype=torch.uint8, device="cuda")
    for dx_is, dy_is in ((0, 1), (2, 3), (0, 3)):
        t = [v.clone() for v in (c.dx_out, c.du, c.x, c.y)]
        out = {"d_" + n: torch.full_like(c.w[n], math.nan) for n in c.w}
        ffi.op_block_norm_bwd(t[2], t[3], t[0], t[1], t[dx_is], t[dy_is], workspace=ws, **c.kw, **out)
        assert torch.equal(t[dx_is], ref["dx"]) and torch.equal(t[dy_is], ref["dy"])
        assert all(torch.equal(out[n], ref[n]) for n in out)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [40, 768, 3000, 9001, 12000])
def test_no_gate_where_each_sequence_would_have_one(kind, d):
    """A description that says gate_per_sequence and holds no gate, for several sequences: the bits of
    one that does not say it."""
    c = Case(BF, F32, 5, 7, d, kind=kind, gate="none")
    got = []
    for per in (0, 1):
        for y in (c.y, None):
            post = y is not None
            w = {n: t if post or not n.startswith("post") else None for n, t in c.w.items()}
            desc, shape, st, dt = ffi._block_desc(c.x, c.du, w["gate"], w["pre_gamma"], w["pre_beta"], w["post_gamma"],
                                                  w["post_beta"], post, None, c.scale, c.eps, kind)
            desc.gate_per_sequence = per
            rows = lambda t, of: ffi._tokens(t, shape, of, "rows")  # noqa: E731, B023
            x_out, u, dx = c.empty(F32), c.empty(BF), c.empty(F32)
            dy = c.empty(BF) if post else None
            lib, stream = ffi.load_library(), torch.cuda.current_stream().cuda_stream
            assert lib.elasto_op_block_norm(desc, rows(c.x, st), rows(y, dt), rows(x_out, st), rows(u, dt), stream) == 0
            sums = {n: torch.full((d,), math.nan, device="cuda") for n in w if w[n] is not None}
            ws = torch.full((ffi.block_norm_workspace(c.x),), 0xff, dtype=torch.uint8, device="cuda")
            place = [sums[n].data_ptr() if n in sums else None
                     for n in ("pre_gamma", "pre_beta", "post_gamma", "post_beta")]
            assert lib.elasto_op_block_norm_bwd(desc, rows(c.x, st), rows(y, dt), rows(c.dx_out, st), rows(c.du, dt),
                                                rows(dx, st), rows(dy, dt), *place, None, ws.data_ptr(), ws.numel(),
                                                stream) == 0
            got.append([x_out, u, dx] + ([dy] if post else []) + list(sums.values()))
    for a, b in zip(got[:2], got[2:]):
        assert len(a) == len(b) and all(torch.equal(x, y) and x.isfinite().all() for x, y in zip(a, b))
    c.check_forward(*got[2][:2])
