"""The factors of an AdamW step, and of a clip, are formed in 64 bits and rounded once."""
import numpy as np
import pytest
import torch

from paper_2106_10796_amd import binding as B

pytestmark = pytest.mark.gpu

PAIRS = [(lr, decay) for lr in (1e-4, 1e-3, 0.0123, 0.1, 0.37, 0.77) for decay in (0.01, 0.1, 0.3, 0.57, 0.9, 1.1, 1.3, 1.7)]


def once(lr, decay):
    return np.float32(1.0 - lr * float(np.float32(decay)))


@pytest.mark.parametrize("bits", [32, 8])
def test_decay(bits):
    """With no gradient and no moments a weight of 1 becomes the factor itself."""
    in_32_bits = [np.float32(1) - np.float32(lr) * np.float32(decay) for lr, decay in PAIRS]
    assert sum(a != once(*p) for a, p in zip(in_32_bits, PAIRS)) >= 5           # pairs that tell the two apart
    state = torch.uint8 if bits == 8 else torch.float32
    for lr in sorted({lr for lr, _ in PAIRS}):
        decays = [d for x, d in PAIRS if x == lr]
        tensors = []
        for d in decays:
            t = dict(weight=torch.ones(300, device="cuda"), grad=torch.zeros(300, device="cuda"), weight_decay=d,
                     m=torch.zeros(300, dtype=state, device="cuda"), v=torch.zeros(300, dtype=state, device="cuda"))
            if bits == 8:
                t |= {s: torch.zeros(B.state_blocks(300), dtype=torch.uint8, device="cuda") for s in ("m_scale", "v_scale")}
            tensors.append(t)
        B.AdamWPlan(tensors, state_bits=bits).step(1, lr)
        for t, d in zip(tensors, decays):
            assert np.array_equal(t["weight"].cpu().numpy(), np.full(300, once(lr, d))), (lr, d)


def test_a_norm_above_the_largest_number():
    """Of finite gradients: infinite in 32 bits, its factor as it is in 64, and the step is skipped; under a scale it is a number again."""
    g, n = 3e38, 1000
    t = dict(weight=torch.ones(n, device="cuda"), grad=torch.full((n,), g, device="cuda"), m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
    plan, out = B.AdamWPlan([t]), torch.zeros(2, device="cuda")
    norm = float(np.float32(g)) * np.sqrt(n)
    plan.grad_norm(out, max_norm=1e30)
    assert out[0].item() == float("inf") and abs(out[1].item() / (1e30 / norm) - 1) < 1e-6
    plan.step(1, 1e-3, clip=out)
    assert bool((t["weight"] == 1).all()) and not t["m"].any() and not t["v"].any()
    plan.grad_norm(out, grad_scale=2.0 ** -100, max_norm=1.0)
    assert abs(out[0].item() / (norm * 2.0 ** -100) - 1) < 1e-6
    plan.step(1, 1e-3, clip=out, grad_scale=2.0 ** -100)
    assert bool((t["weight"] < 1).all()) and bool((t["m"] > 0).all())
