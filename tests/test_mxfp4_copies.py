"""Matrices made of integers that are not uint8: copies, looked over, and never the place of a result."""
import pytest
import torch

from paper_2106_10796_amd import binding as B


def of(dtype, device="cpu"):
    return torch.arange(128).to(dtype).view(2, 64).to(device), torch.full((1, 2, 4), 127, dtype=torch.uint8, device=device)


@pytest.mark.parametrize("dtype", [torch.int16, torch.int32, torch.int64])
def test_bytes_in_wider_integers_are_copied(dtype):
    codes, scales = of(dtype)
    q = B.Mxfp4(codes, scales, 2, 128)
    assert isinstance(q, B.Mxfp4) and q.codes.dtype == torch.uint8 and torch.equal(q.codes.to(dtype), codes) and q.scales is scales
    assert (q.rows, q.cols) == (2, 128)


@pytest.mark.parametrize("bad", [-1, 256, 300])
@pytest.mark.parametrize("which", [0, 1])
def test_integers_that_are_not_bytes_are_refused(bad, which):
    both = [t.short() for t in of(torch.uint8)]
    both[which].view(-1)[-1] = bad
    with pytest.raises(ValueError, match="codes" if which == 0 else "scales"):
        B.Mxfp4(*both, 2, 128)


def test_nothing_is_quantised_into_a_copy():
    x, q = torch.zeros(2, 128), B.Mxfp4(*of(torch.int64), 2, 128)
    room = B.new_mxfp4(2, 128, device="cpu")
    with pytest.raises(TypeError, match="row holds copies"):
        B.cdsgd_mxfp4_quantize(x, q)
    with pytest.raises(TypeError, match="col holds copies"):
        B.cdsgd_mxfp4_quantize(x, room, q)


@pytest.mark.gpu
def test_on_the_gpu():
    codes, scales = of(torch.int64, "cuda")
    q, plain = B.Mxfp4(codes, scales, 2, 128), B.Mxfp4(codes.to(torch.uint8), scales, 2, 128)
    x = torch.ones(2, 128, device="cuda")
    for kw in (dict(row=q), dict(col=B.Mxfp4(torch.zeros(128, 64, dtype=torch.int32, device="cuda"), torch.zeros(1, 128, 4, dtype=torch.uint8,
                                                                                                             device="cuda"), 128, 2))):
        with pytest.raises(TypeError, match="holds copies"):
            B.cdsgd_mxfp4_quantize(x, **kw)
    got = []
    for m in (q, plain):
        out, y = torch.zeros(2, 128, device="cuda"), torch.zeros(2, 2, device="cuda")
        B.cdsgd_mxfp4_dequantize(m, out)
        B.cdsgd_mxfp4_matmul(m, m, y)
        got.append((out, y))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(got[0][1].any())
