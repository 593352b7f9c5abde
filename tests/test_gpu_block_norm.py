"""The norms around a block on the GPU, forward and backward, against a plain implementation in 64 bits.

Tolerances count roundings, with u half a step of a result's type and U that of fp32.  h_out is formed in 64 bits: u + U of itself.  r and n: one rounding.
y: three products (8 U) and u.  Sums over a row in fp32 pass through at most 64 additions, so that a mean is off by 70 U of the mean magnitude
(its products' roundings included); sums over rows through rows / 1024 + 4 additions before they are joined in 64 bits."""
import itertools

import pytest
import torch

from paper_2106_10796_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
KINDS = [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")]


def near(got, want, error, what):
    u = torch.finfo(got.dtype).eps / 2
    error = error * (1 + u) + u * want.abs() + LEAST[got.dtype]
    ok = (got.double() - want).abs() <= error
    assert bool(ok.all()), "%s: %d of %d, first at %s: got %r, want %r within %r" % (
        what, int((~ok).sum()), ok.numel(), (~ok).nonzero()[0].tolist(), float(got[~ok][0]), float(want[~ok][0]), float(error.expand_as(want)[~ok][0]))


class Case:
    """Inputs, outputs with rows further apart than they are long, and the checks."""

    def __init__(self, rows, cols, stream="f32", dtype="bf16", post=True, gate=True, block=True, scale=0.7, eps=1e-6, seed=0, size=1.0):
        self.rows, self.cols, self.block, self.scale, self.eps = rows, cols, block, scale, eps
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.pad = cols % 3
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731

        def wide(t, f=1.0):
            x = torch.full((rows, cols + self.pad), float("nan"), dtype=TYPES[t], device="cuda")
            x[:, :cols] = rnd(rows, cols) * f
            return x[:, :cols]
        self.h, self.b = wide(stream, 3.0 * size), wide(dtype, 0.5 * size) if block else None
        self.dy, self.dh_out = wide(dtype), wide(stream)
        vector = lambda: 1 + 0.3 * rnd(cols)  # noqa: E731
        self.w, self.w_b, self.gate = vector(), vector() if post and block else None, vector() - 1 if gate and block else None
        self.norm = B.BlockNorm(self.w, self.w_b, self.gate, scale, eps)
        self.h_out, self.y = (wide(stream) if block else None), wide(dtype)
        self.dh, self.db = wide(stream), wide(dtype) if block else None
        self.rstd = torch.full((2, rows), 7.0, device="cuda")
        self.dw, self.dw_b, self.dgate = (None if t is None else torch.empty_like(t) for t in (self.w, self.w_b, self.gate))
        self.room = B.new_block_norm_workspace(rows, cols)

    def forward(self, h8=None, b8=None):
        self.norm.forward(self.h, self.y, self.rstd, block=self.b, h_out=self.h_out, h8=h8, block8=b8)

    def saved(self):
        return self.h_out if self.block else self.h

    def backward(self, h=None, b=None, dh_out=True):
        self.norm.backward(self.dy, self.saved() if h is None else h, self.rstd, self.dh, self.dw, self.room, dh_out=self.dh_out if dh_out else None,
                           block=self.b if b is None else b, dblock=self.db, dblock_weight=self.dw_b, dgate=self.dgate)

    def factor(self):
        one = torch.ones(self.cols, dtype=torch.float64, device="cuda")
        return self.scale * (one if self.gate is None else self.gate.double()) * (one if self.w_b is None else self.w_b.double())

    def check_forward(self):
        h = self.h.double()
        if self.block:
            b = self.b.double()
            n = 1 / (b.square().mean(1, keepdim=True) + self.eps).sqrt() if self.w_b is not None else 1.0
            h = h + self.factor() * b * n
            near(self.h_out, h, U * h.abs(), "h_out")
        if self.w_b is not None:
            near(self.rstd[1], n[:, 0], 0 * n[:, 0], "n")
        else:
            assert bool((self.rstd[1] == 7.0).all())
        r = 1 / (h.square().mean(1, keepdim=True) + self.eps).sqrt()
        near(self.rstd[0], r[:, 0], U * r[:, 0], "r")
        y = h * r * self.w.double()
        near(self.y, y, 8 * U * y.abs(), "y")

    def check_backward(self, h, b=None, dh_out=True):
        """At h and b in 64 bits, with the rstd that the forward pass left."""
        r, n = self.rstd[0].double()[:, None], self.rstd[1].double()[:, None] if self.w_b is not None else 1.0
        dy, w, mean = self.dy.double(), self.w.double(), lambda t: t.mean(1, keepdim=True)
        x, g = h * r, dy * w
        c1, off1 = mean(g * x), 70 * U * mean((g * x).abs())
        into = self.dh_out.double() if dh_out else torch.zeros_like(g)
        t = into + r * (g - x * c1)
        off_t = r * (6 * U * (g.abs() + (x * c1).abs()) + x.abs() * off1) + 2 * U * into.abs() + U * t.abs()
        near(self.dh, t, off_t, "dh")
        many = (self.rows / 1024 + 8) * U
        near(self.dw, (dy * x).sum(0), many * (dy * x).abs().sum(0), "dw")
        if not self.block:
            return
        f, c = self.factor(), b * n
        e, off_e = t * f, off_t * f.abs() + 4 * U * (t * f).abs()
        if self.w_b is None:
            near(self.db, e, off_e, "db")
        else:
            c2, off2 = mean(e * c), 70 * U * mean((e * c).abs()) + mean(off_e * c.abs())
            db = n * (e - c * c2)
            near(self.db, db, n * (off_e + c.abs() * off2 + 6 * U * (e.abs() + (c * c2).abs())), "db")
        total, off = (t * c).sum(0), ((off_t + many * t.abs()) * c.abs()).sum(0)
        if self.w_b is not None:
            k = self.scale * (1.0 if self.gate is None else self.gate.double())
            near(self.dw_b, total * k, off * abs(k), "dw_b")
        if self.gate is not None:
            k = self.scale * (1.0 if self.w_b is None else self.w_b.double())
            near(self.dgate, total * k, off * abs(k), "dgate")


def double(t):
    return None if t is None else t.double()


def of(q):
    out = torch.empty(q.rows, q.cols, device="cuda")
    B.cdsgd_mxint8_dequantize(q, out)
    return out.double()


@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 31), (3, 64), (5, 257), (33, 512), (7, 1000), (1030, 65), (3, 2049), (2500, 96), (4, 4096), (3, 5000),
                                       (2, 8193), (2, 16384)])
@pytest.mark.parametrize("stream,dtype", KINDS)
def test_shapes_and_types(rows, cols, stream, dtype):
    c = Case(rows, cols, stream, dtype, seed=rows + cols)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward(double(c.h_out), double(c.b))


@pytest.mark.parametrize("post,gate,block", [(1, 1, 1), (1, 0, 1), (0, 1, 1), (0, 0, 1), (0, 0, 0)])
@pytest.mark.parametrize("dh_out", [True, False])
@pytest.mark.parametrize("rows,cols", [(40, 300), (9, 4100)])
def test_parts(post, gate, block, dh_out, rows, cols):
    c = Case(rows, cols, "f32", "bf16", post, gate, block, seed=cols)
    c.forward()
    c.check_forward()
    c.backward(dh_out=dh_out)
    c.check_backward(double(c.saved()), double(c.b), dh_out)


@pytest.mark.parametrize("stream,dtype", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (20, 33), (6, 2049), (1100, 300)])
def test_saved_in_8_bits(stream, dtype, rows, cols):
    """The saved forms are those of cdsgd_mxint8_quantize, and the backward pass takes either form of each."""
    c = Case(rows, cols, stream, dtype, seed=3)
    c.forward()
    whole = [t.clone() for t in (c.h_out, c.y, c.rstd)]
    h8, b8 = B.new_mxint8(rows, cols), B.new_mxint8(rows, cols)
    c.forward(h8, b8)
    assert all(torch.equal(a, b) for a, b in zip(whole, (c.h_out, c.y, c.rstd)))
    for q, t in ((h8, c.h_out), (b8, c.b)):
        want = B.new_mxint8(rows, cols)
        B.cdsgd_mxint8_quantize(t, want)
        assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    for h, b in itertools.product((None, h8), (None, b8)):
        c.backward(h, b)
        c.check_backward(double(c.h_out) if h is None else of(h), double(c.b) if b is None else of(b))


def test_saved_in_8_bits_without_a_block():
    c = Case(70, 1000, block=False)
    h8 = B.new_mxint8(70, 1000)
    c.forward(h8)
    c.check_forward()
    want = B.new_mxint8(70, 1000)
    B.cdsgd_mxint8_quantize(c.h, want)
    assert torch.equal(h8.codes, want.codes) and torch.equal(h8.scales, want.scales)
    c.backward(h8)
    c.check_backward(of(h8))


@pytest.mark.parametrize("size", [1e-20, 1e-6, 1e15, 1e18])
def test_sizes(size):
    """Squares that fp32 does not hold; eps keeps what is far below it small."""
    c = Case(5, 700, "f32", "f32", size=size, seed=1)
    c.forward()
    c.check_forward()


def test_zeros_and_rows_that_are_not_finite():
    c = Case(6, 500, "f32", "bf16", seed=2)
    c.h[1], c.b[1] = 0, 0
    c.b[3, 7] = float("nan")
    c.h[4, 499] = float("inf")
    c.forward()
    assert bool((c.y[1] == 0).all()) and bool((c.h_out[1] == 0).all())
    assert bool(torch.isnan(c.y[3]).all()) and bool(torch.isnan(c.h_out[3]).all()) and bool(torch.isnan(c.y[4, 499]))
    assert bool(torch.isfinite(c.y[[0, 1, 2, 5]]).all())


def test_same_bits_and_rows_for_themselves():
    """A row's results do not depend on the rows beside it, and a second run gives the same bits, sums over rows included."""
    runs = []
    for _ in range(2):
        c = Case(2100, 1000, seed=9)
        c.forward()
        c.backward()
        runs.append(c)
    a, b = runs
    for name in ("h_out", "y", "rstd", "dh", "db", "dw", "dw_b", "dgate"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    for name in ("h", "b", "dy", "dh_out"):
        setattr(b, name, getattr(b, name)[1500:1501])
    for name in ("h_out", "y", "dh", "db"):
        setattr(b, name, torch.empty_like(getattr(b, name)[:1]))
    b.rstd = torch.empty(2, 1, device="cuda")
    b.forward()
    b.backward()
    assert all(torch.equal(getattr(a, name)[1500:1501], getattr(b, name)) for name in ("h_out", "y", "dh", "db"))


def test_other_streams_and_a_graph():
    c, other = Case(70, 1000, seed=1), Case(70, 1000, seed=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    outs = ("h_out", "y", "rstd", "dh", "db", "dw", "dw_b", "dgate")
    with torch.cuda.stream(side):
        c.forward()
        c.backward()
        with torch.cuda.graph(graph, stream=side):
            c.forward()
            c.backward()
        for k in range(3):
            for name in ("h", "b", "dy", "dh_out"):
                getattr(c, name).copy_(getattr(other, name) * (k + 1))
            graph.replay()
            got = {name: getattr(c, name).clone() for name in outs}
            for name in outs:
                getattr(c, name).fill_(3.0)
            c.forward()
            c.backward()
            side.synchronize()
            assert all(torch.equal(got[name], getattr(c, name)) for name in outs)


def test_gradients_against_differences():
    """The formula that the checks above hold the kernels to is the derivative of the forward formula: central differences in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float64, device="cuda", generator=gen)  # noqa: E731
    h, b, dy, dt, w, w_b, gate = rnd(3, 7), rnd(3, 7), rnd(3, 7), rnd(3, 7), rnd(7), rnd(7), rnd(7)
    rms = lambda x: 1 / (x.square().mean(1, keepdim=True) + 1e-3).sqrt()  # noqa: E731

    def loss(h, b, w, w_b, gate):
        out = h + 0.7 * gate * w_b * b * rms(b)
        return float((out * dt).sum() + (out * rms(out) * w * dy).sum())
    out, n = h + 0.7 * gate * w_b * b * rms(b), rms(b)
    r = rms(out)
    x, g, c, mean = out * r, dy * w, b * n, lambda t: t.mean(1, keepdim=True)
    t = dt + r * (g - x * mean(g * x))
    e = t * 0.7 * gate * w_b
    want = [t, n * (e - c * mean(e * c)), (dy * x).sum(0), 0.7 * gate * (t * c).sum(0), 0.7 * w_b * (t * c).sum(0)]
    args = [h, b, w, w_b, gate]
    for which in range(5):
        for at in range(args[which].numel()):
            d = torch.zeros_like(args[which])
            d.view(-1)[at] = 1e-5
            up, down = ([v + s * d if i == which else v for i, v in enumerate(args)] for s in (1, -1))
            assert abs((loss(*up) - loss(*down)) / 2e-5 - float(want[which].view(-1)[at])) < 1e-7
