"""The two ways in which the binding marshals its calls, in native code and by ctypes, take and refuse the same arguments."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_block_together import Declines

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "ctypes"])
def way(request, monkeypatch):
    B._native()
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_calls", Declines())


@pytest.mark.parametrize("shape", [(1, 3), (3, 1), (1, 3, 1)], ids=str)
def test_starts_are_vectors(way, shape):
    q, k = torch.zeros(9, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(9, 2, 64, dtype=torch.bfloat16, device="cuda")
    starts = torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.zeros(4, 9, device="cuda")
    room = B.new_attention_workspace(q, k, seqs=2, train=True)
    for name in ("starts", "starts_k"):
        bad = {"starts": starts, "starts_k": starts, name: starts.view(shape)}
        with pytest.raises(TypeError, match="%s must be a contiguous CUDA vector of int32" % name):
            B.cdsgd_attention_forward(q, k, k.clone(), out, lse, **bad, workspace=room)
        with pytest.raises(TypeError, match="%s must be a contiguous CUDA vector of int32" % name):
            B.cdsgd_attention_backward(out, q, k, k.clone(), out.clone(), lse, q.clone(), k.clone(), k.clone(), **bad, workspace=room)
