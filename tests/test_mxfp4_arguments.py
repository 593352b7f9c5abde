"""What is no matrix in MXFP4 is named, in every place that takes one."""
import pytest
import torch

from paper_2106_10796_amd import binding as B


@pytest.mark.parametrize("other", [None, torch.zeros(2, 64, dtype=torch.uint8), (1, 2, 3, 4), 5], ids=["None", "tensor", "tuple", "number"])
def test_no_matrix(other, monkeypatch):
    q, y = B.new_mxfp4(2, 128, device="cpu"), torch.zeros(2, 2)
    with pytest.raises(TypeError, match="a must be an Mxfp4"):
        B.cdsgd_mxfp4_matmul(other, q, y)
    with pytest.raises(TypeError, match="q must be an Mxfp4"):
        B.cdsgd_mxfp4_dequantize(other, y)
    monkeypatch.setattr(B, "_dev", lambda *a: 16)            # (as if a's buffers were on the GPU; the library is not reached)
    with pytest.raises(TypeError, match="b must be an Mxfp4"):
        B.cdsgd_mxfp4_matmul(q, other, y)
