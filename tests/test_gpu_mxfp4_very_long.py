"""Matrices in MXFP4 of more rows than one launch of a wave to every few of them holds."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_ops_long import give_back, random_codes, some_rows, values  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K", [(1, 128), (16, 100), (20, 128)])
def test_product_of_few_rows(M, K):
    long = (1 << 28) + 37
    gen = torch.Generator(device="cuda").manual_seed(M)
    a, b = B.Mxfp4(*random_codes(M, 1, gen), M, K), B.Mxfp4(*random_codes(long, 1, gen), long, K)
    a.codes[:, K // 2:] = 0                                         # what is behind the end is 0
    out = torch.empty(M, long, dtype=torch.bfloat16, device="cuda")
    B.cdsgd_mxfp4_matmul(a, b, out)
    at = torch.tensor([0, 1, 63, 64, 2 ** 26 - 1, 2 ** 26, 2 ** 27 + 5, 2 ** 28 - 1, 2 ** 28, long - 38, long - 2, long - 1], device="cuda")
    few, other = values(some_rows(b, at)), values(a)
    want, size = other @ few.t().contiguous(), other.abs() @ few.abs().t().contiguous()
    # sums under one pair of scales are exact, those of the four blocks of 32 are rounded once each, and the result once to 16 bits
    assert bool(((out[:, at].double() - want).abs() <= 12 * 2.0 ** -24 * size + 2.0 ** -8 * want.abs()).all())


def on_the_grid(shape, dtype, seed):
    """Values that MXFP4 holds exactly; blocks of 32 along the last axis begin with a 4."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda").to(dtype)[torch.randint(0, 8, shape, dtype=torch.uint8, device="cuda", generator=gen).int()]
    x[..., ::32] = 4
    return x


def test_rows_there_and_back():
    x = on_the_grid(((1 << 28) + 37, 3), torch.float16, 1)
    q = B.new_mxfp4(*x.shape)
    B.cdsgd_mxfp4_quantize(x, q)
    out = torch.zeros_like(x)
    B.cdsgd_mxfp4_dequantize(q, out)
    assert torch.equal(out, x)


def test_columns_there_and_back():
    x = on_the_grid((1, (1 << 29) + 37), torch.float32, 2).t().contiguous()
    q = B.new_mxfp4(1, x.shape[0])
    B.cdsgd_mxfp4_quantize(x, None, q)
    out = torch.zeros(1, x.shape[0], device="cuda")
    B.cdsgd_mxfp4_dequantize(q, out)
    assert torch.equal(out.t(), x)
