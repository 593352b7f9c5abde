"""Matrices and lists whose bytes pass 2^32: the far end is what the same rows give by themselves."""
import pytest
import torch

from paper_2106_10796_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def random_codes(rows, g, gen):
    codes = torch.randint(0, 256, (rows, 64 * g), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.randint(120, 128, (g, rows, 4), dtype=torch.uint8, device="cuda", generator=gen)
    return codes, scales


def some_rows(q, rows):
    return B.Mxfp4(q.codes[rows].contiguous(), q.scales[:, rows].contiguous(), len(rows), q.cols)


def values(q):
    out = torch.empty(q.rows, q.cols, device="cuda")
    B.cdsgd_mxfp4_dequantize(q, out)
    return out.double()


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("which", ["a", "b"])
def test_product(M, which):
    """(the places of the sampled rows cover both sides of byte 2^32 of the codes, and for `a` of the result)"""
    gen = torch.Generator(device="cuda").manual_seed(M)
    g, long = 65, 1100000
    K = 128 * g
    big, small = B.Mxfp4(*random_codes(long, g, gen), long, K), B.Mxfp4(*random_codes(M, g, gen), M, K)
    a, b = (big, small) if which == "a" else (small, big)
    out = torch.empty(a.rows, b.rows, device="cuda")
    B.cdsgd_mxfp4_matmul(a, b, out, B.new_mxfp4_workspace([(a.rows, b.rows, K)]))
    edge = 2 ** 32 // (64 * g)
    at = torch.tensor([0, 1, 77, edge - 1, edge, edge + 1, 2 ** 20, long - 257, long - 2, long - 1], device="cuda")
    few, other = values(some_rows(big, at)), values(small)
    want, size = few @ other.t().contiguous(), few.abs() @ other.abs().t().contiguous()
    got = (out[at] if which == "a" else out[:, at].t()).double()
    # sums under one pair of scales are exact, those of the blocks of 32 are rounded once each
    assert bool(((got - want).abs() <= (K / 32 + 8) * 2.0 ** -24 * size + 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("rows,cols", [(300000, 8200), (520, 4800000)])
def test_quantisation_and_values(rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, dtype=torch.bfloat16, device="cuda", generator=gen)
    assert x.numel() * 2 > 2 ** 32
    row, col = B.new_mxfp4(rows, cols), B.new_mxfp4(cols, rows)
    B.cdsgd_mxfp4_quantize(x, row, col)
    alone = B.new_mxfp4(rows, cols)
    B.cdsgd_mxfp4_quantize(x, alone)
    assert torch.equal(row.codes, alone.codes) and torch.equal(row.scales, alone.scales)
    # the last rows and the last columns by themselves, from the start of a block on
    r0, c0 = (rows - 70) // 128 * 128, (cols - 70) // 128 * 128
    low, right = B.new_mxfp4(rows - r0, cols), B.new_mxfp4(cols - c0, rows)
    B.cdsgd_mxfp4_quantize(x[r0:].contiguous(), low)
    B.cdsgd_mxfp4_quantize(x[:, c0:].contiguous(), None, right)
    assert torch.equal(row.codes[r0:], low.codes) and torch.equal(row.scales[:, r0:], low.scales)
    assert torch.equal(col.codes[c0:], right.codes) and torch.equal(col.scales[:, c0:], right.scales)
    back, part = torch.empty_like(x), torch.empty(rows - r0, cols, dtype=x.dtype, device="cuda")
    B.cdsgd_mxfp4_dequantize(row, back)
    B.cdsgd_mxfp4_dequantize(low, part)
    assert torch.equal(back[r0:], part) and bool((back[:1].float() - x[:1].float()).abs().max() < 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_norm(bits):
    n = 2 ** 31 + 5
    first = n // 4096 * 4096 - 16 * 4096                           # the end by itself
    gen = torch.Generator(device="cuda").manual_seed(bits)

    def of(weight, grad):
        k = weight.numel()
        state = lambda: torch.zeros(k, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda")  # noqa: E731
        t = dict(weight=weight, grad=grad, m=state(), v=state())
        if bits == 8:
            t |= {s: torch.zeros(B.state_blocks(k), dtype=torch.uint8, device="cuda") for s in ("m_scale", "v_scale")}
        return t

    w = torch.randn(n, device="cuda", generator=gen)
    g = torch.randn(n, dtype=torch.bfloat16, device="cuda", generator=gen)
    whole, end = of(w, g), of(w[first:].clone(), g[first:].clone())
    plan = B.AdamWPlan([whole], grad_dtype=torch.bfloat16, state_bits=bits)
    out = torch.empty(2, device="cuda")
    plan.grad_norm(out)
    want = sum(float(g[i:i + 2 ** 28].double().square().sum()) for i in range(0, n, 2 ** 28)) ** 0.5
    assert abs(float(out[0]) - want) <= 2 * 2.0 ** -24 * want
    plan.step(1, 1e-2)
    B.AdamWPlan([end], grad_dtype=torch.bfloat16, state_bits=bits).step(1, 1e-2)
    assert torch.equal(w[first:], end["weight"])
    if bits == 32:
        assert torch.equal(whole["m"][first:], end["m"]) and torch.equal(whole["v"][first:], end["v"])
        return
    # the dither goes by the element's number in the list: codes differ by one at most
    for s, magnitude in (("m", 127), ("v", 255)):
        assert torch.equal(whole[s + "_scale"][first // 256:], end[s + "_scale"])
        a, b = whole[s][first:].int(), end[s].int()
        assert bool(((a & magnitude) - (b & magnitude)).abs().max() <= 1)
