"""The norms around a block on the GPU: what is rounded, rows that are not finite, and groups that go through several rows, against 64 bits."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_block_norm import TYPES

pytestmark = pytest.mark.gpu


def nearest(x, dtype):
    """x, in 64 bits, rounded once to a 16-bit type: of the numbers beside the one that two roundings give, the nearest, of two the even one."""
    near = x.float().to(dtype)
    bits = near.view(torch.int16)
    best, distance = near, (near.double() - x).abs()
    for step in (-1, 1):
        other = (bits + step).view(dtype)
        d = (other.double() - x).abs()
        take = (d < distance) | ((d == distance) & (other.view(torch.int16) % 2 == 0))
        best, distance = torch.where(take, other, best), torch.where(take, d, distance)
    return best


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cols", [64, 1000, 5000])
@pytest.mark.parametrize("scale", [1 + 2.0 ** -40, 1 - 2.0 ** -40, 1.0])
def test_h_out_is_rounded_once(dtype, cols, scale):
    """h plus half a step of it, times just above and just below 1: a sum in fp32 would lie halfway between two numbers of the type."""
    t, u = TYPES[dtype], torch.finfo(TYPES[dtype]).eps
    gen = torch.Generator(device="cuda").manual_seed(cols)
    h = (1 + torch.randint(0, int(1 / u), (9, cols), device="cuda", generator=gen) * u).to(t)
    b = torch.full_like(h, u / 2)
    h[:, ::2], b[:, ::2] = -h[:, ::2], -b[:, ::2]
    h_out, y, rstd = torch.empty_like(h), torch.empty_like(h), torch.empty(2, 9, device="cuda")
    B.BlockNorm(torch.ones(cols, device="cuda"), scale=scale).forward(h, y, rstd, block=b, h_out=h_out)
    want = nearest(h.double() + b.double() * scale, t)
    assert torch.equal(h_out, want), (h_out != want).nonzero()[0]
