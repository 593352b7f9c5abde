"""What stands between the products of a transformer block in training, as cases that can be timed and compared: attention over
packed sequences, the norms around a block with its gate and residual scale, gated activations, and activations held in
8 bits for the backward pass.

One pass of a case:

  attention  out = softmax(scale q k^T) v for every sequence of a packed batch, with the logarithm of each row's sum; query heads share
             key heads in groups; where `causal` says so, query i of a sequence sees the keys up to i + (keys - queries).  `held` is how
             many keys each sequence has before its first query's.  With `train` the gradients of q, k and v too.
  norm       the end of one block and the beginning of the next: h' = h + scale * gate * norm(b) * block weight, y = norm(h') * weight,
             both root-mean-square norms.  With `train` the gradients of h, b and the three weights, from the saved h' and b: as they
             are, or (`bits` 8) in 8 bits, which the forward pass leaves.
  gated      y = act(a) * u.  With `train` the gradients of a and u, from the saved a and u as above.
  held8      a matrix to 8 bits and back

Where `own` is false a pass computes the operators from elementary torch operations in 32 bits; where it is true it makes the calls of
`paper_2106_10796_amd.binding`.

8 bits are the MXINT8 of the OCP Microscaling Formats specification 1.0: 32 values in a row share a power of two, that of the largest
magnitude among them, and a value is a whole number of 64ths of it, at most 127, rounded to nearest, ties to even.  Codes are [rows, 32 g]
with g = ceil(cols / 32), scale bytes (exponent + 127) [rows, g].
"""
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _attention_case(name, **more):
    c = {"name": name, "kind": "attention", "seqs": 1, "tokens": 1, "held": 0, "heads": 1, "kv": 1, "dim": 128, "causal": 1, "x": "bf16",
         "train": 0}
    c.update(more)
    return c


def _rows_case(name, kind, **more):
    c = {"name": name, "kind": kind, "m": 1, "n": 1, "x": "bf16", "bits": 16, "train": 0}
    if kind == "norm":
        c.update({"stream": "f32", "post": 1, "gate": 1})
    if kind == "gated":
        c.update({"act": "silu"})
    c.update(more)
    return c


def listed():
    return [
        # a short question to a small model: latency only
        _attention_case("attention_17_tokens", tokens=17, heads=8, kv=2, dim=64),
        # one new token after a long text
        _attention_case("attention_token_32k", tokens=1, held=32767, heads=32, kv=8),
        # the ordinary training batch: texts of different lengths, packed
        _attention_case("attention_train_packed", seqs=8, tokens=8191, heads=32, kv=8, train=1),
        # an encoder's batch, both directions, heads of their own
        _attention_case("attention_train_f16", seqs=16, tokens=7999, heads=12, kv=12, dim=64, causal=0, x="f16", train=1),
        # the largest: a long text read at once
        _attention_case("attention_16k", tokens=16384, heads=16, kv=2),
        # a single token between two blocks
        _rows_case("norm_token", "norm", n=4096),
        # the ordinary training step: 32-bit stream, 16-bit blocks
        _rows_case("norm_train_8192", "norm", m=8192, n=4096, train=1),
        # an odd matrix with its stream in 16 bits, a gate but no norm after the block, saved in 8 bits
        _rows_case("norm8_train_odd", "norm", m=1003, n=2049, x="f16", stream="f16", post=0, bits=8, train=1),
        # a few tokens
        _rows_case("gated_16_tokens", "gated", m=16, n=8192),
        # the widest activations of a training step, saved in 8 bits
        _rows_case("gated8_train_8192", "gated", m=8192, n=16384, bits=8, train=1),
        # a block's output, saved for the backward pass and read back there
        _rows_case("held8_8192", "held8", m=8192, n=4096),
        # an odd matrix in 32 bits
        _rows_case("held8_odd", "held8", m=1003, n=2049, x="f32"),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(lo * (hi / lo) ** rng.random()))
        return v if rng.random() < 0.6 else max(8, v // 64 * 64) if v >= 64 else v

    kind = rng.choice(["attention", "attention", "attention", "norm", "norm", "gated", "gated", "held8"])
    if kind == "attention":
        kv = rng.choice([1, 2, 4, 8])
        c = _attention_case("", heads=kv * rng.choice([1, 2, 4, 8]), kv=kv, dim=rng.choice([40, 64, 64, 80, 96, 128, 128, 128]),
                            causal=int(rng.random() < 0.7), x=rng.choice(["bf16", "bf16", "f16"]), train=int(rng.random() < 0.6),
                            seqs=size(1, 64), tokens=size(65, 8192))
        if rng.random() < 0.25:
            # the next piece of a text, or a few new tokens of each of several
            c["held"], c["train"] = size(16, 8192), 0
            c["tokens"] = min(c["tokens"], 1024)
        c["tokens"] = max(c["tokens"], c["seqs"])
        # what a plain pass over padded sequences takes stays below that of the largest listed case
        while c["heads"] * c["seqs"] * max(_lengths(c)) * (max(_lengths(c)) + c["held"]) > 1 << 30:
            c["tokens"], c["seqs"] = max(c["tokens"] * 2 // 3, 1), max(c["seqs"] * 2 // 3, 1)
            c["tokens"] = max(c["tokens"], c["seqs"])
    else:
        more = {"x": rng.choice(["bf16", "bf16", "f16", "f32"]), "m": size(1, 8192), "n": size(33, 16384)}
        if kind == "norm":
            more["stream"] = rng.choice(["f32", more["x"]])
            more["post"], more["gate"] = rng.choice([(1, 1), (1, 0), (0, 1), (0, 0)])
            more["n"] = size(65, 8192)
        if kind == "gated":
            more["act"] = rng.choice(["silu", "silu", "gelu_tanh"])
        if kind != "held8":
            more["train"] = int(rng.random() < 0.7)
            more["bits"] = rng.choice([8, 16]) if more["train"] else 16
        c = _rows_case("", kind, **more)
    return {k: v for k, v in c.items() if k != "name"}


def _lengths(case):
    """Queries of each sequence: unequal, in an order that is neither rising nor falling."""
    n, total = case["seqs"], case["tokens"]
    share = [2 + (5 * i + 3) % 7 for i in range(n)]
    ends = [sum(share[:i + 1]) * (total - n) // sum(share) + i + 1 for i in range(n)]
    return [b - a for a, b in zip([0] + ends, ends)]


def work(case):
    b = BYTES[case["x"]]
    if case["kind"] == "attention":
        pairs = 0
        for q in _lengths(case):
            pairs += q * (q + case["held"]) - (q * (q - 1) // 2 if case["causal"] else 0)
        keys = case["tokens"] + case["seqs"] * case["held"]
        q, kv = case["tokens"] * case["heads"] * case["dim"] * b, keys * case["kv"] * case["dim"] * b
        lse, flops = case["tokens"] * case["heads"] * 4, 4 * case["dim"] * pairs * case["heads"]
        # forward: q, k, v in, out and lse out; backward: the gradient of out in, those of q, k and v out
        return {"bytes": 2 * q + 2 * kv + lse + (2 * q + 2 * kv if case["train"] else 0), "flops": flops * (7 if case["train"] else 2) / 2}
    n = case["m"] * case["n"]
    if case["kind"] == "held8":
        return {"bytes": n * (2 * b + 33 / 32), "flops": 4 * n}
    if case["kind"] == "gated":
        # the 8-bit forms are written and read by different calls
        saved = 2 * 33 / 32 if case["bits"] == 8 else 0
        return {"bytes": n * (3 * b + (saved + 3 * b + (saved or 2 * b) if case["train"] else 0)), "flops": n * (30 if case["train"] else 10)}
    s = BYTES[case["stream"]]
    forward, backward = n * (2 * s + 2 * b), n * (2 * s + 2 * b + (2 * 33 / 32 if case["bits"] == 8 else s + b))
    saved = n * 2 * 33 / 32 if case["bits"] == 8 else 0
    return {"bytes": forward + (saved + backward if case["train"] else 0) + 4 * case["n"] * 3, "flops": n * (30 if case["train"] else 10)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 29)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    like = torch.empty_like
    t = DTYPE[case["x"]]
    state = {"case": case}
    if case["kind"] == "attention":
        lens = _lengths(case)
        held, heads, kv, dim = case["held"], case["heads"], case["kv"], case["dim"]
        T, K = case["tokens"], case["tokens"] + case["seqs"] * held
        starts = lambda add: torch.tensor([sum(lens[:i]) + i * add for i in range(len(lens) + 1)], dtype=torch.int32).cuda()  # noqa: E731
        state["starts"], state["starts_k"] = starts(0), starts(held)
        # logits of a trained model spread over a few units, and some channels of the keys are far larger than the others
        state["q"] = (normal(T, heads, dim) * 1.5).to(t)
        state["k"] = (normal(K, kv, dim) * (1 + 3 * (torch.rand(kv, dim, device="cuda", generator=gen) < 0.02))).to(t)
        state["v"] = normal(K, kv, dim).to(t)
        state["out"], state["lse"] = like(state["q"]), torch.empty(heads, T, device="cuda")
        if case["train"]:
            # gradients in fp16 come with a loss scale
            state["dout"] = (normal(T, heads, dim) * (0.1 if case["x"] == "f16" else 1e-3)).to(t)
            state |= {"d" + n: like(state[n]) for n in "qkv"}
        if own:
            from paper_2106_10796_amd import binding
            state["room"] = binding.new_attention_workspace(state["q"], state["k"], seqs=case["seqs"], train=bool(case["train"]))
        return state
    m, n = case["m"], case["n"]
    # some channels far larger than the others, as activations have them
    channel = 1 + 15 * (torch.rand(n, device="cuda", generator=gen) < 0.01)
    if case["kind"] == "held8":
        state["x"] = (normal(m, n) * channel).to(t)
        state["back"] = like(state["x"])
        names = {"x8"}
    elif case["kind"] == "gated":
        state["a"], state["u"] = (normal(m, n) * 2).to(t), (normal(m, n) * channel).to(t)
        state["y"] = like(state["a"])
        if case["train"]:
            state["dy"] = (normal(m, n) * (0.1 if case["x"] == "f16" else 1e-3)).to(t)
            state["da"], state["du"] = like(state["a"]), like(state["a"])
        names = {"a8", "u8"}
    else:
        s = DTYPE[case["stream"]]
        state["h"], state["b"] = (normal(m, n) * channel).to(s), (normal(m, n) * 0.5).to(t)
        state["h_out"], state["y"], state["rstd"] = like(state["h"]), like(state["b"]), torch.empty(2, m, device="cuda")
        state["w"] = 1 + 0.1 * normal(n)
        state["w_b"] = 1 + 0.1 * normal(n) if case["post"] else None
        state["gate"] = 0.5 + 0.1 * normal(n) if case["gate"] else None
        state["scale"] = 0.7
        if case["train"]:
            size = 0.1 if case["x"] == "f16" else 1e-3
            state["dy"], state["dh_out"] = (normal(m, n) * size).to(t), (normal(m, n) * size).to(s)
            state["dh"], state["db"] = like(state["h"]), like(state["b"])
            state |= {"d" + k: None if state[k] is None else like(state[k]) for k in ("w", "w_b", "gate")}
        names = {"h8", "b8"}
        if own:
            from paper_2106_10796_amd import binding
            state["norm"] = binding.BlockNorm(state["w"], block_weight=state["w_b"], gate=state["gate"], scale=state["scale"], eps=EPS)
            if case["train"]:
                state["room"] = binding.new_block_norm_workspace(m, n)
    if own and (case["bits"] == 8 or case["kind"] == "held8"):
        from paper_2106_10796_amd import binding
        state |= {name: binding.new_mxint8(m, n) for name in sorted(names)}
    return state


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _padded(x, starts, longest):
    """[seqs, longest, ...] of a packed x, 0 behind a sequence's end, and which rows are rows of a sequence."""
    at = torch.arange(longest, device=x.device)
    inside = at < (starts[1:] - starts[:-1])[:, None]
    rows = (starts[:-1, None] + at).clamp(max=x.shape[0] - 1).long()
    return x[rows].float() * inside[:, :, None, None], inside


def _packed(x, starts, tokens):
    """The rows of a padded x [seqs, longest, ...] one after the other."""
    t = torch.arange(tokens, device=x.device)
    seq = torch.searchsorted(starts[1:].contiguous(), t.int(), right=True)
    return x[seq, t - starts[seq]]


def _plain_attention(state):
    case = state["case"]
    kv, group, dim = case["kv"], case["heads"] // case["kv"], case["dim"]
    B, T, longest = case["seqs"], case["tokens"], max(_lengths(case))
    keys = longest + case["held"]
    scale = dim ** -0.5

    def by_head(x):
        """[seqs, kv, group * longest, dim] of [seqs, longest, heads, dim]."""
        return x.view(B, longest, kv, group, dim).permute(0, 2, 3, 1, 4).reshape(B, kv, group * longest, dim)

    q, _ = _padded(state["q"], state["starts"], longest)
    k, inside = _padded(state["k"], state["starts_k"], keys)
    v, _ = _padded(state["v"], state["starts_k"], keys)
    q, k, v = by_head(q), k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    hidden = ~inside[:, None, :]
    if case["causal"]:
        i, j = torch.arange(longest, device=q.device), torch.arange(keys, device=q.device)
        hidden = hidden | (j > i[:, None] + case["held"])
    s.view(B, kv, group, longest, keys).masked_fill_(hidden[:, None, None], float("-inf"))
    most = s.amax(3, keepdim=True)
    p = s.sub_(most).exp_()
    total = p.sum(3, keepdim=True)
    p.div_(total)
    o = torch.matmul(p, v)
    lse = (most + total.log()).view(B, case["heads"], longest).transpose(1, 2)
    state["out"].copy_(_packed(o.view(B, kv, group, longest, dim).permute(0, 3, 1, 2, 4).reshape(B, longest, case["heads"], dim),
                               state["starts"], T))
    state["lse"].copy_(_packed(lse, state["starts"], T).t())
    outs = {"out": state["out"], "lse": state["lse"]}
    if case["train"]:
        do, _ = _padded(state["dout"], state["starts"], longest)
        do = by_head(do)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
        ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(3, keepdim=True)).mul_(p).mul_(scale)
        dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
        dq = torch.matmul(ds, k)
        dq = dq.view(B, kv, group, longest, dim).permute(0, 3, 1, 2, 4).reshape(B, longest, case["heads"], dim)
        state["dq"].copy_(_packed(dq, state["starts"], T))
        for name, d in (("dk", dk), ("dv", dv)):
            state[name].copy_(_packed(d.transpose(1, 2), state["starts_k"], state["k"].shape[0]))
            outs[name] = state[name]
        outs["dq"] = state["dq"]
    return outs


def _eight_bits(x):
    """The values of x in 8 bits, as 32-bit floats."""
    rows, cols = x.shape
    g = -(-cols // 32)
    p = torch.zeros(rows, g * 32, dtype=torch.float32, device=x.device)
    p[:, :cols] = x
    p = p.view(rows, g, 32)
    # the exponent field of the largest magnitude; a 64th of it needs more than 32 bits where it is small.  (The power of two is put together
    # from its bits: torch.exp2 is not exact on the GPU, and 16-bit values often lie halfway between two codes.)
    e = ((p.abs().amax(2, keepdim=True).view(torch.int32) >> 23) & 0xFF).long()
    step = ((e + (1023 - 133)) << 52).view(torch.float64)
    codes = (p.double() / step).round().clamp(-127, 127)
    return (codes * step).float().view(rows, g * 32)[:, :cols]


def _plain_held8(state):
    state["back"].copy_(_eight_bits(state["x"]))
    return state["back"]


def _act(a, kind):
    """act(a) and its slope."""
    if kind == "silu":
        s = 1 / (1 + torch.exp(-a))
        return a * s, s * (1 + a * (1 - s))
    c = 0.7978845608028654
    t = torch.tanh(c * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * c * (1 + 3 * 0.044715 * a * a)


def _plain_gated(state):
    case = state["case"]
    a, u = state["a"].float(), state["u"].float()
    state["y"].copy_(_act(a, case["act"])[0] * u)
    if not case["train"]:
        return state["y"]
    if case["bits"] == 8:
        a, u = _eight_bits(state["a"]), _eight_bits(state["u"])
    act, slope = _act(a, case["act"])
    dy = state["dy"].float()
    state["da"].copy_(dy * u * slope)
    state["du"].copy_(dy * act)
    return {"y": state["y"], "da": state["da"], "du": state["du"]}


def _plain_norm(state):
    case, scale = state["case"], state["scale"]
    # in 64 bits: what is saved of it in 8 bits may lie next to the border of two codes
    b, w = state["b"].double(), state["w"]
    n = 1 / (b.square().mean(1, keepdim=True) + EPS).sqrt() if case["post"] else 1.0
    into = (state["gate"].double() if case["gate"] else 1.0) * (state["w_b"].double() if case["post"] else 1.0) * scale
    h = state["h"].double() + into * (b * n)
    state["h_out"].copy_(h)
    h, n, into = h.float(), n.float() if case["post"] else 1.0, into.float() if case["post"] or case["gate"] else into
    r = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    state["y"].copy_(h * r * w)
    outs = {"h_out": state["h_out"], "y": state["y"]}
    if not case["train"]:
        return outs
    held = _eight_bits if case["bits"] == 8 else torch.Tensor.float
    x, c, dy = held(state["h_out"]) * r, held(state["b"]) * n, state["dy"].float()
    g = dy * w
    t = state["dh_out"].float() + r * (g - x * (g * x).mean(1, keepdim=True))
    state["dh"].copy_(t)
    e = t * into
    state["db"].copy_(n * (e - c * (e * c).mean(1, keepdim=True)) if case["post"] else e)
    # long sums
    total = (t.double() * c).sum(0)
    state["dw"].copy_((dy.double() * x).sum(0))
    if case["post"]:
        state["dw_b"].copy_(total * scale * (state["gate"] if case["gate"] else 1.0))
    if case["gate"]:
        state["dgate"].copy_(total * scale * (state["w_b"] if case["post"] else 1.0))
    return outs | {k: state[k] for k in ("dh", "db", "dw", "dw_b", "dgate") if state[k] is not None}


# ---------------------------------------------------------------------------
# a pass
# ---------------------------------------------------------------------------
def _own_attention(state):
    from paper_2106_10796_amd import binding
    case = state["case"]
    lens = dict(starts=state["starts"], starts_k=state["starts_k"], causal=bool(case["causal"]))
    binding.cdsgd_attention_forward(state["q"], state["k"], state["v"], state["out"], state["lse"], workspace=state["room"], **lens)
    outs = {"out": state["out"], "lse": state["lse"]}
    if case["train"]:
        binding.cdsgd_attention_backward(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["dq"], state["dk"],
                                         state["dv"], workspace=state["room"], **lens)
        outs |= {"dk": state["dk"], "dv": state["dv"], "dq": state["dq"]}
    return outs


def _own_held8(state):
    from paper_2106_10796_amd import binding
    binding.cdsgd_mxint8_quantize(state["x"], state["x8"])
    binding.cdsgd_mxint8_dequantize(state["x8"], state["back"])
    return state["back"]


def _own_gated(state):
    from paper_2106_10796_amd import binding
    case = state["case"]
    a8, u8 = state.get("a8"), state.get("u8")
    binding.cdsgd_gated_forward(state["a"], state["u"], state["y"], a8, u8, act=case["act"])
    if not case["train"]:
        return state["y"]
    saved = (state["a"], state["u"]) if a8 is None else (a8, u8)
    binding.cdsgd_gated_backward(state["dy"], *saved, state["da"], state["du"], act=case["act"])
    return {"y": state["y"], "da": state["da"], "du": state["du"]}


def _own_norm(state):
    norm, h8, b8 = state["norm"], state.get("h8"), state.get("b8")
    norm.forward(state["h"], state["y"], state["rstd"], block=state["b"], h_out=state["h_out"], h8=h8, block8=b8)
    outs = {"h_out": state["h_out"], "y": state["y"]}
    if not state["case"]["train"]:
        return outs
    saved = (state["h_out"], state["b"]) if h8 is None else (h8, b8)
    norm.backward(state["dy"], saved[0], state["rstd"], state["dh"], state["dw"], state["room"], dh_out=state["dh_out"], block=saved[1],
                  dblock=state["db"], dblock_weight=state["dw_b"], dgate=state["dgate"])
    return outs | {k: state[k] for k in ("dh", "db", "dw", "dw_b", "dgate") if state[k] is not None}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attention": _own_attention, "held8": _own_held8, "gated": _own_gated, "norm": _own_norm}[kind](state)
    return {"attention": _plain_attention, "held8": _plain_held8, "gated": _plain_gated, "norm": _plain_norm}[kind](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_attention(case, state):
    """One sequence and one key head after the other; gradients by differentiation of the forward pass."""
    lens, held, group = _lengths(case), case["held"], case["heads"] // case["kv"]
    outs = {"out": torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda"),
            "lse": torch.zeros(state["lse"].shape, dtype=torch.float64, device="cuda")}
    if case["train"]:
        outs |= {"d" + n: torch.zeros(state[n].shape, dtype=torch.float64, device="cuda") for n in "kvq"}
    first_q = first_k = 0
    for n in lens:
        rows, cols = slice(first_q, first_q + n), slice(first_k, first_k + n + held)
        for head in range(case["kv"]):
            mine = slice(head * group, (head + 1) * group)
            with torch.set_grad_enabled(bool(case["train"])):
                q = state["q"][rows, mine].double().transpose(0, 1).contiguous().requires_grad_(bool(case["train"]))
                k = state["k"][cols, head].double().contiguous().requires_grad_(bool(case["train"]))
                v = state["v"][cols, head].double().contiguous().requires_grad_(bool(case["train"]))
                logits = torch.matmul(q, k.t()) / case["dim"] ** 0.5
                if case["causal"]:
                    seen = torch.ones(n, n + held, dtype=torch.bool, device="cuda").tril(held)
                    logits = torch.where(seen, logits, torch.full_like(logits[:1, :1, :1], float("-inf")))
                lse = torch.logsumexp(logits, 2)
                o = torch.matmul(torch.exp(logits - lse[:, :, None]), v)
                if case["train"]:
                    dq, dk, dv = torch.autograd.grad(o, (q, k, v), state["dout"][rows, mine].double().transpose(0, 1))
                    outs["dq"][rows, mine], outs["dk"][cols, head], outs["dv"][cols, head] = dq.transpose(0, 1), dk, dv
            outs["out"][rows, mine], outs["lse"][mine, rows] = o.detach().transpose(0, 1), lse.detach()
            del logits, lse, o, q, k, v
        first_q, first_k = first_q + n, first_k + n + held
    return outs


def _exact_held8(x):
    """Block by block as the format's specification has it."""
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    whole = x.shape[1] // 32 * 32
    for lo, hi in ((0, whole), (whole, x.shape[1])):
        if lo < hi:
            part = x[:, lo:hi].double()
            part = part.reshape(part.shape[0], -1, min(32, hi - lo))
            _, e = torch.frexp(part.abs().amax(-1, keepdim=True))
            step = torch.tensor([2.0 ** (k - 6) for k in range(-127, 128)], dtype=torch.float64, device="cuda")[(e - 1).clamp(min=-127).long() + 127]
            out[:, lo:hi] = ((part / step).round().clamp(-127, 127) * step).reshape(part.shape[0], -1)
    return out


def _exact_gated(case, state):
    def y_of(a, u):
        if case["act"] == "silu":
            return a * torch.sigmoid(a) * u
        return a * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (a + 0.044715 * a ** 3)) * u

    y = y_of(state["a"].double(), state["u"].double())
    if not case["train"]:
        return y
    held = _exact_held8 if case["bits"] == 8 else torch.Tensor.double
    a, u = held(state["a"]).requires_grad_(), held(state["u"]).requires_grad_()
    da, du = torch.autograd.grad(y_of(a, u), (a, u), state["dy"].double())
    return {"y": y, "da": da, "du": du}


def _exact_norm(case, state):
    """The gradient of x / rms(x) is r (1 - x x^T r^2 / n), at the saved x and the forward pass's r = 1 / rms(x)."""
    d = lambda name: state[name].double()  # noqa: E731
    rms = lambda x: 1 / (x.pow(2).mean(1, keepdim=True) + EPS).sqrt()  # noqa: E731
    gate = d("gate") if case["gate"] else torch.ones((), dtype=torch.float64, device="cuda")
    w_b = d("w_b") if case["post"] else torch.ones((), dtype=torch.float64, device="cuda")
    n = rms(d("b")) if case["post"] else torch.ones(case["m"], 1, dtype=torch.float64, device="cuda")
    h = d("h") + state["scale"] * gate * w_b * n * d("b")
    r = rms(h)
    outs = {"h_out": h, "y": h * r * d("w")}
    if not case["train"]:
        return outs
    saved_h, saved_b = h.to(DTYPE[case["stream"]]), state["b"]
    if case["bits"] == 8:
        saved_h, saved_b = _exact_held8(saved_h), _exact_held8(saved_b)
    saved_h, saved_b = saved_h.double(), saved_b.double()
    m = case["n"]
    gy = d("dy") * d("w")
    dh = d("dh_out") + r * gy - saved_h * r ** 3 * (gy * saved_h).sum(1, keepdim=True) / m
    de = dh * state["scale"] * gate * w_b
    db = n * de - saved_b * n ** 3 * (de * saved_b).sum(1, keepdim=True) / m if case["post"] else de
    outs |= {"dh": dh, "db": db, "dw": (d("dy") * saved_h * r).sum(0)}
    if case["post"]:
        outs["dw_b"] = (dh * state["scale"] * gate * saved_b * n).sum(0)
    if case["gate"]:
        outs["dgate"] = (dh * state["scale"] * w_b * saved_b * n).sum(0)
    return outs


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "attention":
        return _exact_attention(case, state)
    if case["kind"] == "held8":
        return _exact_held8(state["x"])
    return _exact_gated(case, state) if case["kind"] == "gated" else _exact_norm(case, state)
