"""Attention's gradients where values, gradients or logits are far from 1, against plain implementations in 64 bits.

Tolerances count roundings as those of test_gpu_attention.py do, but that dS of fp16 tensors is off by at most 2^-32 of the largest |dS| that it is summed
up with, a row's for dq and a key's for dk: its power of two brings the largest so far to 2^7 at least, and half a step of fp16's smallest numbers is 2^-25."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_attention import SMALL, U, check_forward, close as close_finite, half_step, inputs, logit_error, probabilities, reference, starts_of, tiny, tiny_p

pytestmark = pytest.mark.gpu


def close(got, want, error, what):
    """fp16 rounds 65520 and more to infinity: an infinity is near where the tolerance reaches a number of its sign that large."""
    if got.dtype == torch.float16:
        past = torch.isinf(got) & (torch.where(got > 0, want, -want) + error >= 65520)
        got = torch.where(past, want, got.double()) if bool(past.any()) else got
    close_finite(got, want, error, what)


def run(dout, q, k, v, lens_q, lens_k, causal, scale):
    room = B.new_attention_workspace(q, k, seqs=len(lens_q), train=True)
    out, lse, grads = torch.empty_like(q), torch.empty(q.shape[1], q.shape[0], device="cuda"), [torch.empty_like(t) for t in (q, k, v)]
    starts = starts_of(lens_q), starts_of(lens_k)
    B.cdsgd_attention_forward(q, k, v, out, lse, *starts, causal, scale, room)
    B.cdsgd_attention_backward(dout, q, k, v, out, lse, *grads, *starts, causal, scale, room)
    return out, lse, grads


def check_gradients(dout, q, k, v, out, lse, grads, lens_q, lens_k, causal, scale, exact_logits=False):
    """exact_logits: the products q . k are exact in fp32, whatever their order, so that what is left of a logit's error is that of differences."""
    u, dim, f16 = half_step(q), q.shape[2], q.dtype == torch.float16
    dq, dk, dv = grads
    for rows, cols, h, mine, s, size, x, y, z in reference(q, k, v, lens_q, lens_k, causal, scale):
        nq, nk = s.shape[1], s.shape[2]
        do, o = (t[rows, mine].double().transpose(0, 1).contiguous() for t in (dout, out))
        at = torch.logsumexp(s, 2) if exact_logits else lse[mine, rows].double()
        p = probabilities(s, at)
        e_p = 2 * U * (8 * torch.where(torch.isinf(s), 0.0, s - at[..., None]).abs() + 16 + nk) if exact_logits else 2 * logit_error(s, size, at, dim)
        dp, delta = torch.matmul(do, z.t().contiguous()), (do * o).sum(2, keepdim=True)
        ds = p * (dp - delta)
        e_ds = ds.abs() * (u + e_p) + 2 * U * dim * p * (torch.matmul(do.abs(), z.abs().t().contiguous()) + (do * o).abs().sum(2, keepdim=True))
        e_ds = e_ds + 2 * SMALL * (1 + (dp - delta).abs())
        least = 2.0 ** -32 * (ds.abs() + e_ds) * (p > 0) if f16 else torch.zeros_like(ds)
        of_row, of_key = least.amax(2, keepdim=True) * (p > 0), least.amax((0, 1), keepdim=True) * (p > 0)
        want = scale * torch.matmul(ds, y)
        close(dq[rows, mine].transpose(0, 1), want, scale * torch.matmul(e_ds + of_row + 2 * U * nk * ds.abs(), y.abs()) + u * want.abs() + tiny(q), "dq")
        n = nq * s.shape[0]
        e_v = p * (u + e_p) + 2 * SMALL + tiny_p(q, 15)
        for got, w, e_w, other, what, f in ((dk, ds, e_ds + of_key, x, "dk", scale), (dv, p, e_v, do, "dv", 1.0)):
            flat = lambda t: t.reshape(n, t.shape[2])  # noqa: E731
            want = f * torch.matmul(flat(w).t().contiguous(), flat(other))
            error = f * torch.matmul((flat(e_w) + 2 * U * n * flat(w).abs()).t().contiguous(), flat(other).abs()) + u * want.abs() + tiny(q)
            close(got[cols, h], want, error, what)


def go(dout, q, k, v, lens_q, lens_k, causal, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out, lse, grads = run(dout, q, k, v, lens_q, lens_k, causal, scale)
    check_gradients(dout, q, k, v, out, lse, grads, lens_q, lens_k, causal, scale)
    return grads


def test_dS_above_the_largest_number_of_fp16():
    """Two keys with values of 1100 and -1100: dS is 70400 and -70400, the gradients ordinary numbers."""
    full = lambda n, x: torch.full((n, 1, 128), x, dtype=torch.float16, device="cuda")  # noqa: E731
    sign = torch.tensor([1.0, -1.0], device="cuda").half()[:, None, None]
    dq, dk, dv = go(full(1, 1.0), full(1, 0.0), full(2, 0.01) * sign, full(2, 1100.0) * sign, [1], [2], False)
    assert bool(torch.isfinite(dq).all()) and float(dq[0, 0, 0]) == pytest.approx(2 * 70400 * float(torch.tensor(0.01).half()) / 128 ** 0.5, rel=2.0 ** -9)
    assert bool((dk == 0).all()) and bool((dv == 0.5).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("v_size,dout_size", [(0.02, 1.0), (0.005, 1e-3), (4e3, 1.0), (4e3, 1e-4), (1.0, 30.0), (1e-4, 1e-4), (2e4, 1.0)])
@pytest.mark.parametrize("causal", [True, False])
def test_values_and_gradients_of_any_size(v_size, dout_size, causal, dim):
    lens = [40, 300]
    q, k, v, dout = inputs(lens, lens, 4, 2, dim, "f16", seed=11)
    go((dout.float() * dout_size).half(), q, k, (v.float() * v_size).clamp(-65504, 65504).half(), lens, lens, causal)


@pytest.mark.parametrize("dim", [64, 128])
def test_dS_of_one_row_and_of_one_key_from_almost_0_to_the_largest(dim):
    """The first tile's probabilities are e^-85 and the last's ordinary, with values and gradients of 3e4: dS from 2^-87 to 2^30 and more in one sum."""
    half = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(15)
    small = lambda n: (torch.randint(-16, 17, (n, 1, dim), device="cuda", generator=gen) * 2.0 ** -24).half()  # noqa: E731
    sign = lambda n: torch.where(torch.arange(n, device="cuda") % 2 == 0, 3e4, -3e4).half()[:, None, None].expand(n, 1, dim).contiguous()  # noqa: E731
    # a row over 64 keys far below and 64 beside 0
    q, k, v, dout = half(40, 1, dim) + 1, torch.cat([half(64, 1, dim) - 85.0 / dim, small(64)]), sign(128), half(40, 1, dim) + 3e4
    go(dout, q, k, v, [40], [128], False, scale=1.0)
    # keys seen by 64 queries from far below and by 64 from beside 0
    q, k, v, dout = torch.cat([half(64, 1, dim) - 85.0 / dim, small(64)]), torch.cat([half(20, 1, dim) + 1, half(20, 1, dim)]), sign(40), half(128, 1, dim) + 3e4
    go(dout, q, k, v, [128], [40], False, scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("v_size", [1.0, 0.02, 0.005])
@pytest.mark.parametrize("keys", [16384, 40000])
def test_flat_rows_of_many_keys(keys, v_size, dtype):
    """Probabilities of 1 over the number of keys: dS of a row is small throughout."""
    q, k, v, dout = inputs([3], [keys], 2, 1, 128, dtype, seed=12)
    go(dout, q * 0.1, k, (v.float() * v_size).to(v.dtype), [3], [keys], False)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("large", [slice(0, 2), slice(150, 152), slice(298, 300)], ids=["first", "middle", "last"])
def test_rows_with_gradients_of_very_different_size(large, dim):
    """A few rows' gradients are 10^6 times the others': a row's results, and those of keys that the large ones do not see, are as if they were alone."""
    lens = [300]
    q, k, v, dout = inputs(lens, lens, 4, 2, dim, "f16", seed=13)
    size = torch.full((300, 1, 1), 1e-4, device="cuda")
    size[large] = 1e2
    go((dout.float() * size).half(), q, k, v, lens, lens, True)


def test_rows_without_gradients():
    """Rows of zeros first, last and between: the first dS that is not 0 sets the power of two."""
    lens = [260]
    q, k, v, dout = inputs(lens, lens, 4, 1, 64, "f16", seed=14)
    for rows in (slice(0, 130), slice(70, 260), slice(0, 260)):
        some = dout.clone()
        some[rows] = 0
        dq, dk, dv = go(some, q, k, v, lens, lens, False)
        assert bool((dq[rows] == 0).all())


def far_case(dtype, dim, scale, sign, lens_q, lens_k, seed, near_rows=()):
    """Logits of scale * 2^10 and a few times scale * 2^-10 beside: products q . k are multiples of 2^-10 below 2^14, so that fp32 holds every partial sum."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, K, heads, kv = sum(lens_q), sum(lens_k), 4, 2
    t = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    ints = lambda n, h: torch.randint(-3, 4, (n, h, dim), device="cuda", generator=gen).float() / 32  # noqa: E731
    q, k = ints(T, heads), ints(K, kv)
    q[:, :, 4:], k[:, :, 4:] = 0, 0
    q[:, :, 0], k[:, :, 0] = 32 * sign, 32
    for rows in near_rows:
        q[rows, :, 0] = 0
    _, _, v, dout = inputs(lens_q, lens_k, heads, kv, dim, dtype, seed=seed)
    return q.to(t), k.to(t), v, dout


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 40])
@pytest.mark.parametrize("scale", [2.0 ** 2, 2.0 ** 3, 2.0 ** 10, 2.0 ** 20, 2.0 ** 30])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("causal", [True, False])
def test_gradients_of_far_logits(causal, sign, scale, dim, dtype):
    """Logits from 2^12 to 2^40, where fp32 has no bits of lse left for what the probabilities are made of, beside rows of ordinary ones."""
    lens = [150, 1, 77]
    q, k, v, dout = far_case(dtype, dim, scale, sign, lens, lens, 21, near_rows=(slice(40, 47), slice(90, 128), slice(160, 190)))
    out, lse, grads = run(dout, q, k, v, lens, lens, causal, scale)
    check_gradients(dout, q, k, v, out, lse, grads, lens, lens, causal, scale, exact_logits=True)


@pytest.mark.parametrize("lens_q,lens_k", [([200, 3], [60, 500]), ([1, 1], [3000, 70])], ids=str)
def test_far_logits_of_rows_that_see_few_keys(lens_q, lens_k):
    """Rows that see nothing among them."""
    q, k, v, dout = far_case("bf16", 64, 2.0 ** 12, 1, lens_q, lens_k, 22)
    out, lse, grads = run(dout, q, k, v, lens_q, lens_k, True, 2.0 ** 12)
    check_gradients(dout, q, k, v, out, lse, grads, lens_q, lens_k, True, 2.0 ** 12, exact_logits=True)


def test_far_logits_of_ordinary_numbers_keep_their_sums():
    """Logits of about 10^6 and 10^9 that fp32 does not hold: probabilities are those of the forward pass, whose sum over keys is 1, so that a dout of one
    number throughout gives dv its sum over queries, and v of one number throughout no dq (but for what `out` was rounded by)."""
    lens = [300]
    for size in (1e3, 3e4):
        q, k, v, _ = inputs(lens, lens, 4, 2, 128, "bf16", seed=23)
        q, k, v, dout = (q.float() * size).bfloat16(), (k.float() * size).bfloat16(), torch.ones_like(v), torch.ones_like(q)
        out, _, (dq, dk, dv) = run(dout, q, k, v, lens, lens, True, 1.0)
        # (sum of P, each rounded by half a step, over their sum: half a step, and the result's rounding)
        assert bool(((out.double() - 1).abs() <= 2 * 2.0 ** -8).all())
        total = dv.double().sum(0)[:, 0]                          # of 300 queries of two heads, each a sum of probabilities: half a step each way
        assert bool(((total - 600).abs() <= 600 * 3 * 2.0 ** -8).all()), total
        assert all(bool(torch.isfinite(t).all()) for t in (dq, dk, dv))


def test_a_sequence_in_other_batches():
    """Where no keys are taken in parts a sequence's results are the same to the bit in any batch, dq among them."""
    lens = [200, 77, 130]
    q, k, v, dout = inputs(lens, lens, 8, 2, 128, "bf16", seed=41)
    a = run(dout, q, k, v, lens, lens, True, 0.1)
    for cut, n in ((slice(0, 200), 200), (slice(200, 277), 77), (slice(277, 407), 130)):
        b = run(*(t[cut].contiguous() for t in (dout, q, k, v)), [n], [n], True, 0.1)
        assert torch.equal(a[0][cut], b[0]) and torch.equal(a[1][:, cut], b[1]) and all(torch.equal(x[cut], y) for x, y in zip(a[2], b[2]))


@pytest.mark.parametrize("others", [[], [64], [64] * 31, [4096, 1]], ids=len)
def test_a_token_over_many_keys_beside_others(others):
    """A new token's keys are taken in as many parts as its batch says: within the tolerances in each, the same from run to run, gradients the same in
    any batch at the same out and lse."""
    gen = torch.Generator(device="cuda").manual_seed(42)
    rnd = lambda n, h: torch.randn(n, h, 128, device="cuda", generator=gen).bfloat16()  # noqa: E731
    q, k, v, dout, seqs = rnd(1, 8), rnd(4096, 2), rnd(4096, 2), rnd(1, 8), 1 + len(others)
    alone = run(dout, q, k, v, [1], [4096], True, 0.1)
    more = sum(others)
    q, k, v, dout = (torch.cat([a, rnd(n, a.shape[1])]) for a, n in ((q, len(others)), (k, more), (v, more), (dout, len(others))))
    lens_q, lens_k = [1] * seqs, [4096, *others]
    out, lse, _ = run(dout, q, k, v, lens_q, lens_k, True, 0.1)
    check_forward(q, k, v, out, lse, lens_q, lens_k, True, 0.1)
    again = run(dout, q, k, v, lens_q, lens_k, True, 0.1)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    out[:1], lse[:, :1] = alone[0], alone[1]
    room, grads = B.new_attention_workspace(q, k, seqs=seqs, train=True), [torch.empty_like(t) for t in (q, k, v)]
    B.cdsgd_attention_backward(dout, q, k, v, out, lse, *grads, starts_of(lens_q), starts_of(lens_k), True, 0.1, room)
    assert all(torch.equal(x[:n], y) for x, y, n in zip(grads, alone[2], (1, 4096, 4096)))


@pytest.mark.parametrize("far", [slice(4990, 5000), slice(0, 3), slice(4200, 4201)], ids=["last", "first", "one"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_few_far_rows_of_many(far, dtype):
    """More tiles of rows than a wave has lanes, of which one has far rows."""
    near = [slice(0, far.start), slice(far.stop, 5000)]
    q, k, v, dout = far_case(dtype, 64, 2.0 ** 10, 1, [5000], [100], 24, near_rows=near)
    out, lse, grads = run(dout, q, k, v, [5000], [100], False, 2.0 ** 10)
    check_gradients(dout, q, k, v, out, lse, grads, [5000], [100], False, 2.0 ** 10, exact_logits=True)
