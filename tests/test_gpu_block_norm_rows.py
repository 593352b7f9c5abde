"""The norms around a block on the GPU: what is rounded, rows that are not finite, and groups that go through several rows, against 64 bits."""
import itertools

import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_block_norm import KINDS, TYPES, Case, double, of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cols", [64, 1000, 5000])
@pytest.mark.parametrize("scale", [1 + 2.0 ** -40, 1 - 2.0 ** -40, 1.0])
def test_h_out_is_rounded_to_fp32_and_then_to_its_type(dtype, cols, scale):
    """h plus half a step of it, times just above and just below 1: a sum that fp32 puts halfway between two numbers of the type."""
    t, u = TYPES[dtype], torch.finfo(TYPES[dtype]).eps
    gen = torch.Generator(device="cuda").manual_seed(cols)
    h = (1 + torch.randint(0, int(1 / u), (9, cols), device="cuda", generator=gen) * u).to(t)
    b = torch.full_like(h, u / 2)
    h[:, ::2], b[:, ::2] = -h[:, ::2], -b[:, ::2]
    h_out, y, rstd = torch.empty_like(h), torch.empty_like(h), torch.empty(2, 9, device="cuda")
    B.BlockNorm(torch.ones(cols, device="cuda"), scale=scale).forward(h, y, rstd, block=b, h_out=h_out)
    want = h.double() + b.double() * scale
    assert torch.equal(h_out, want.float().to(t)) and torch.equal(h_out, want.to(t))


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("stream,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("cols", [70, 1500, 6000])
def test_rows_that_are_not_finite_go_as_the_formulas_do(cols, stream, dtype, post):
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda t: torch.randn(6, cols, device="cuda", generator=gen).to(TYPES[t])  # noqa: E731
    h, b = rnd(stream), rnd(dtype)
    inf, nan, last = float("inf"), float("nan"), cols - 1
    h[1, last], h[2, 3], b[3, last], b[4, 5] = -inf, nan, inf, nan
    h_out, y, rstd, w = torch.empty_like(h), torch.empty_like(b), torch.empty(2, 6, device="cuda"), torch.ones(cols, device="cuda")
    B.BlockNorm(w, w.clone() if post else None).forward(h, y, rstd, block=b, h_out=h_out)
    x = b.double()
    if post:
        x = x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt()
    want_h = h.double() + x
    want_y = want_h / (want_h.square().mean(1, keepdim=True) + 1e-6).sqrt()
    for got, want in ((h_out, want_h), (y, want_y)):
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert bool(torch.isnan(y[1, last])) and bool((y[1, :last] == 0).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[4]).all())
    assert bool(torch.isnan(y[3]).all()) if post else bool(torch.isnan(y[3, last])) and bool((y[3, :last] == 0).all())
    assert bool(torch.isfinite(y[[0, 5]]).all())


# For every width's shape of a group more rows than there are groups in a launch (4096 over a group's waves forward, backward 2^21 over the columns and a
# quarter of the rows at most), so that groups go from row to row, some of them once more than others.
LONG = [(4500, 200), (2100, 500), (1100, 1000), (1100, 1500), (1100, 2049), (1100, 4096), (1100, 5000), (1030, 8192), (600, 8200), (530, 12289), (515, 16384)]


@pytest.mark.parametrize("rows,cols", LONG)
@pytest.mark.parametrize("stream,dtype", KINDS)
def test_groups_of_several_rows(rows, cols, stream, dtype):
    c = Case(rows, cols, stream, dtype, seed=rows + cols)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward(double(c.h_out), double(c.b))


@pytest.mark.parametrize("rows,cols", LONG)
@pytest.mark.parametrize("post,gate,block,dh_out", [(1, 0, 1, 1), (0, 1, 1, 0), (0, 0, 1, 1), (0, 0, 0, 1), (0, 0, 0, 0)])
def test_parts_of_several_rows(rows, cols, post, gate, block, dh_out):
    c = Case(rows, cols, "f32", "bf16", post, gate, block, seed=cols)
    c.forward()
    c.check_forward()
    c.backward(dh_out=bool(dh_out))
    c.check_backward(double(c.saved()), double(c.b), dh_out)


@pytest.mark.parametrize("rows,cols", [(2100, 500), (1100, 2049), (1100, 5000), (600, 8200), (515, 16384)])
@pytest.mark.parametrize("stream,dtype", KINDS)
def test_several_rows_saved_in_8_bits(rows, cols, stream, dtype):
    c = Case(rows, cols, stream, dtype, seed=5)
    h8, b8 = B.new_mxint8(rows, cols), B.new_mxint8(rows, cols)
    c.forward(h8, b8)
    c.check_forward()
    for q, t in ((h8, c.h_out), (b8, c.b)):
        want = B.new_mxint8(rows, cols)
        B.cdsgd_mxint8_quantize(t, want)
        assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    for h, b in itertools.product((None, h8), (None, b8)):
        c.backward(h, b)
        c.check_backward(double(c.h_out) if h is None else of(h), double(c.b) if b is None else of(b))
