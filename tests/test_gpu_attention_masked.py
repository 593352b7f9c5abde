"""NaN and infinities in tokens that `causal` hides: what does not see them is what it was without them, to the bit, in both passes."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_attention import inputs
from test_gpu_attention_range import far_case, run

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), float("-inf")]


def step(q, k, v, dout, lens_q, lens_k, scale):
    out, lse, (dq, dk, dv) = run(dout, q, k, v, lens_q, lens_k, True, scale)
    return {"out": out, "lse": lse.t(), "dq": dq, "dk": dk, "dv": dv}


def check(q, k, v, dout, lens_q, lens_k, tokens, scale=None, heads=None):
    """tokens: numbers of keys (of the last sequence) that are hit one after the other, and queries at the same place."""
    scale = q.shape[2] ** -0.5 if scale is None else scale
    group, kv = q.shape[1] // k.shape[1], k.shape[1] - 1
    clean = step(q, k, v, dout, lens_q, lens_k, scale)
    first_q, first_k, more = sum(lens_q[:-1]), sum(lens_k[:-1]), lens_k[-1] - lens_q[-1]
    mine = slice(kv * group, None)
    assert all(bool(torch.isfinite(t).all()) for name, t in clean.items() if name != "lse")     # (that is -infinity where there is no key)
    for n, at in enumerate(tokens):
        bad = BAD[n % 3]
        for t in (k, v):
            was = t[first_k + at, kv].clone()
            t[first_k + at, kv, (5 * n) % q.shape[2]] = bad
            got = step(q, k, v, dout, lens_q, lens_k, scale)
            t[first_k + at, kv] = was
            hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
            hit[first_q + max(at - more, 0):, mine] = True
            for name in ("out", "lse", "dq"):
                assert torch.equal(got[name][~hit], clean[name][~hit]), (name, at, bad)
            for name in ("dk", "dv"):
                assert torch.equal(got[name][:first_k], clean[name][:first_k]) and torch.equal(got[name][:, :kv], clean[name][:, :kv]), (name, at, bad)
            assert bool((~torch.isfinite(got["out"][hit])).any()) or not bool(hit.any()) or t is k
        row = at - more
        if 0 <= row < lens_q[-1]:
            head = q.shape[1] - 1 - n % group
            for t in (q, dout):
                was = t[first_q + row, head].clone()
                t[first_q + row, head, (3 * n) % q.shape[2]] = bad
                got = step(q, k, v, dout, lens_q, lens_k, scale)
                t[first_q + row, head] = was
                hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
                hit[first_q + row, head] = True
                for name in ("out", "lse", "dq"):
                    assert torch.equal(got[name][~hit], clean[name][~hit]), (name, at, bad)
                seen = torch.zeros(k.shape[:2], dtype=torch.bool, device="cuda")
                seen[first_k:first_k + at + 1, kv] = True
                for name in ("dk", "dv"):
                    assert torch.equal(got[name][~seen], clean[name][~seen]), (name, at, bad)
                assert bool((~torch.isfinite(got["dk"][seen])).any())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (4, 2, 128), (8, 1, 40), (40, 1, 128), (6, 2, 96), (70, 2, 64)])
def test_prompts(dtype, heads, kv, dim):
    lens = [130, 300]
    q, k, v, dout = inputs(lens, lens, heads, kv, dim, dtype, seed=31)
    check(q, k, v, dout, lens, lens, [0, 1, 31, 32, 63, 64, 100, 129, 191, 255, 298, 299])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens_q,lens_k", [([5], [700]), ([9, 100], [3, 170]), ([40, 33], [400, 20])], ids=str)
def test_pieces_of_a_prompt(lens_q, lens_k, dtype):
    """More keys than queries, the keys of the first split over groups, and fewer."""
    q, k, v, dout = inputs(lens_q, lens_k, 8, 2, 64, dtype, seed=32)
    n = lens_k[-1]
    check(q, k, v, dout, lens_q, lens_k, [0, n // 2, n - 34 if n > 34 else 1, n - 3, n - 2, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_beside_far_logits(dtype):
    lens = [150]
    q, k, v, dout = far_case(dtype, 64, 2.0 ** 3, 1, lens, lens, 33, near_rows=(slice(40, 60),))
    check(q, k, v, dout, lens, lens, [0, 31, 45, 63, 70, 149], scale=2.0 ** 3)


def test_several_at_once():
    """Infinities of both signs and NaN in keys, values, queries and gradients of one tile: every row has what it sees of them."""
    lens = [96]
    q, k, v, dout = inputs(lens, lens, 2, 1, 64, "bf16", seed=34)
    clean = step(q, k, v, dout, lens, lens, 0.125)
    inf = float("inf")
    v[50, 0, 3], v[60, 0, 3], v[60, 0, 9] = inf, -inf, -inf
    got = step(q, k, v, dout, lens, lens, 0.125)
    assert torch.equal(got["out"][:50], clean["out"][:50])
    assert bool((got["out"][50:60, :, 3] == inf).all()) and bool(torch.isnan(got["out"][60:, :, 3]).all()) and bool((got["out"][60:, :, 9] == -inf).all())
    rest = [i for i in range(64) if i not in (3, 9)]
    assert torch.equal(got["out"][:, :, rest], clean["out"][:, :, rest]) and torch.equal(got["out"][:60, :, 9], clean["out"][:60, :, 9])
