"""The training step's other operators as cases that can be timed and compared: AdamW over a layer list with states in 32
or in 8 bits, the norm of a list's gradients, and microscaled 4-bit floating point (MXFP4): quantisation and products.

One pass of a case:

  adamw     clip by the list's gradient norm where `clip` says so, then one AdamW step over the list.  With states in 8
            bits the step is followed by what a program does that looks at them or saves them: both read out in 16 bits.
  norm      the norm of a list's gradients and the factor that brings it down to `max_norm`
  quantize  a matrix to MXFP4 in blocks along its rows (`row`), down its columns (`col`) or both, each read back
  product   A[m, k] times B[n, k] transposed, both in MXFP4
  linear    a linear layer on activations in 16 bits against weights that are kept in MXFP4: the input quantised and
            multiplied and, where `train` says so, both gradients, each a product of operands quantised along the axis
            that it sums over

Where `own` is false a pass computes the operators from elementary torch operations in 32 bits; where it is true it
makes the calls of `paper_2106_10796_amd.binding`.

What is held in few bits, as both sides read and write it:

  states in 8 bits  blocks of 256 elements.  A block's scale byte b is the exponent field of its largest magnitude as a
            32-bit float.  The first moment has a sign, 4 exponent and 3 mantissa bits, the second 5 and 3: with T = 14
            and T = 30 the code is what remains of the 32-bit pattern of |x| 2^(T - b) after a dither has been added
            below its last bit and 20 bits have been shifted out.  A second moment above 0 keeps a code of 1 at least.
  dither    16 bits for each of the two moments from a hash of the call's seed and the element's number in the list,
            in which every tensor begins at a multiple of 256.
  MXFP4     blocks of 32 elements, 4-bit values 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, a block's scale 2^(s - 127).  Codes
            [rows, 64 g] with g = ceil(cols / 128), two to a byte, the first in the low half; scale bytes [g, rows, 4].

Layer lists are those of the models that the package's synthetic workloads are shaped after, as slices of one arena for
each kind of buffer.  Matrix sizes are those of the same models' fully connected layers, with batches from one token on.
"""
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                      # elements under one scale of an 8-bit state
TOP_M, TOP_V = 14, 30            # exponent field that a block's largest magnitude is brought to
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _conv(cout, cin, k):
    return cout * cin * k * k


def _layers(case):
    """Elements of each tensor of the case's list."""
    if case["layers"] == "flat":
        return [case["n"]]
    if case["layers"] == "resnet20":
        sizes, cin = [_conv(16, 3, 3), 16, 16], 16
        for c in (16, 32, 64):
            for b in range(3):
                sizes += [_conv(c, cin, 3), c, c, _conv(c, c, 3), c, c]
                if b == 0 and cin != c:
                    sizes += [_conv(c, cin, 1), c, c]
                cin = c
        return sizes + [640, 10]
    if case["layers"] == "resnet50":
        sizes, cin = [_conv(64, 3, 7), 64, 64], 64
        for blocks, w in ((3, 64), (4, 128), (6, 256), (3, 512)):
            for b in range(blocks):
                sizes += [_conv(w, cin, 1), w, w, _conv(w, w, 3), w, w, _conv(4 * w, w, 1), 4 * w, 4 * w]
                if b == 0:
                    sizes += [_conv(4 * w, cin, 1), 4 * w, 4 * w]
                cin = 4 * w
        return sizes + [2048 * 1000, 1000]
    if case["layers"] == "vgg16":
        sizes, cin = [], 3
        for c in (64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512):
            sizes += [_conv(c, cin, 3), c]
            cin = c
        for a, b in ((25088, 4096), (4096, 4096), (4096, 1000)):
            sizes += [a * b, b]
        return sizes
    # mixed: a matrix and a vector in turn, up to `n` elements in all
    sizes, left, a = [], case["n"], max(case["n"] // 5, 1)
    while left > 0 and len(sizes) < 60:
        for s in (a, max(a // 997, 1)):
            s = min(s, left)
            if s:
                sizes.append(s)
            left -= s
        a = max(a * 3 // 4, 1)
    return sizes


def _list_case(name, kind, layers, **more):
    c = {"name": name, "kind": kind, "layers": layers, "n": 0, "grad": "f32", "bits": 32, "clip": 0, "copy": 0}
    c.update(more)
    return c


def _matrix_case(name, kind, **more):
    c = {"name": name, "kind": kind, "m": 1, "n": 1, "k": 1, "x": "bf16", "out": "bf16", "row": 1, "col": 0, "train": 0}
    c.update(more)
    return c


def listed():
    return [
        # the step of a small model, 65 tensors in one launch: latency only
        _list_case("adamw_resnet20", "adamw", "resnet20"),
        # the ordinary mixed-precision step: 16-bit gradients, clipped, 32-bit states, and the 16-bit weights of the next pass
        _list_case("adamw_resnet50_bf16", "adamw", "resnet50", grad="bf16", clip=1, copy=1),
        # the same list with states in 8 bits, gradients in fp16
        _list_case("adamw8_resnet50_f16", "adamw", "resnet50", grad="f16", bits=8),
        # a large model with states in 8 bits
        _list_case("adamw8_vgg16_bf16", "adamw", "vgg16", grad="bf16", bits=8, clip=1, copy=1),
        # the largest: the norm of a 1 GiB bucket of 32-bit gradients with an odd end
        _list_case("norm_bucket_256m", "norm", "flat", n=(1 << 28) - 3),
        # activations of a few tokens on their way into a product
        _matrix_case("quantize_16_tokens", "quantize", m=16, n=4096),
        # the master weights of a large layer after a step, for the forward and for the backward pass
        _matrix_case("quantize_fc1_both", "quantize", m=4096, n=25088, x="f32", col=1),
        # an odd matrix, fp16
        _matrix_case("quantize_odd_both", "quantize", m=1003, n=2049, x="f16", col=1),
        # one token through a large layer
        _matrix_case("product_token", "product", m=1, n=4096, k=25088),
        # a batch through a classifier, 32-bit logits
        _matrix_case("product_batch64", "product", m=64, n=1000, k=4096, out="f32"),
        # the ordinary large product
        _matrix_case("product_8192_tokens", "product", m=8192, n=4096, k=4096),
        # forward and both gradients of a large layer
        _matrix_case("linear_train_2048", "linear", m=2048, n=4096, k=25088, train=1),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(lo * (hi / lo) ** rng.random()))
        return v if rng.random() < 0.6 else max(8, v // 64 * 64) if v >= 64 else v

    kind = rng.choice(["adamw", "adamw", "adamw", "norm", "quantize", "quantize", "product", "product", "product", "linear", "linear"])
    if kind in ("adamw", "norm"):
        more = {"grad": rng.choice(["f32", "bf16", "bf16", "f16"]), "n": size(1 << 11, 1 << 26) + rng.randrange(4)}
        if kind == "adamw":
            more["bits"], more["clip"] = rng.choice([32, 8]), rng.randrange(2)
            more["copy"] = rng.randrange(2) if more["grad"] != "f32" else 0
        return {k: v for k, v in _list_case("", kind, rng.choice(["flat", "mixed", "mixed"]), **more).items() if k != "name"}
    more = {"x": rng.choice(["bf16", "bf16", "f16", "f32"]), "out": rng.choice(["bf16", "f32", "f16"])}
    if kind == "quantize":
        more["row"], more["col"] = rng.choice([(1, 0), (0, 1), (1, 1), (1, 1)])
        more["m"], more["n"] = size(1, 8192), size(33, 12000)
    else:
        more["m"] = size(1, 2048) if rng.random() < 0.7 else rng.randrange(1, 17)
        more["n"], more["k"] = size(129, 8192), size(65, 8192)
        if kind == "linear":
            more["train"] = rng.randrange(2)
            more["x"] = rng.choice(["bf16", "f16"])
            more["out"] = more["x"]
    return {k: v for k, v in _matrix_case("", kind, **more).items() if k != "name"}


def _groups(cols):
    return -(-cols // 128)


def work(case):
    if case["kind"] in ("adamw", "norm"):
        n, g = sum(_layers(case)), BYTES[case["grad"]]
        if case["kind"] == "norm":
            return {"bytes": n * g, "flops": 2 * n}
        # weights in and out, gradient, states in and out, the 16-bit copy, states read out in 16 bits
        each = 8 + g + (16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4) + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": n * (14 + 2 * case["clip"])}
    m, n, k, out = case["m"], case["n"], case["k"], BYTES[case["out"]]
    held = lambda rows, cols: rows * cols * 17 / 32  # noqa: E731
    if case["kind"] == "quantize":
        forms = case["row"] + case["col"]
        return {"bytes": m * n * BYTES[case["x"]] + forms * (held(m, n) + m * n * BYTES[case["x"]]), "flops": 3 * forms * m * n}
    if case["kind"] == "product":
        return {"bytes": held(m, k) + held(n, k) + m * n * out, "flops": 2 * m * n * k}
    x = BYTES[case["x"]]
    bytes_, flops = m * k * x + held(n, k) + m * n * x, 2 * m * n * k
    if case["train"]:
        bytes_, flops = bytes_ + m * n * x + held(k, n) + m * k * x + n * k * 4, 3 * flops
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _e8m0(device):
    """What a scale byte stands for."""
    return torch.tensor([2.0 ** (s - 127) for s in range(255)] + [float("nan")], dtype=torch.float64, device=device).float()


def _spread(values, sizes):
    """One number for each tensor, as a column over the arena's blocks."""
    blocks = torch.tensor([-(-s // BLOCK) for s in sizes])
    return torch.repeat_interleave(torch.tensor(values, dtype=torch.float32), blocks).cuda()[:, None]


def _prepare_list(case, gen):
    sizes = _layers(case)
    first, total = [], 0
    for s in sizes:
        first.append(total)
        total += -(-s // BLOCK) * BLOCK
    # what lies between two tensors of the arena is no part of the list, and 0
    inside = torch.zeros(total + 1, dtype=torch.int8, device="cuda")
    ends = torch.tensor([f + s for f, s in zip(first, sizes)], device="cuda")
    inside[torch.tensor(first, device="cuda")] += 1
    inside[ends] -= 1
    inside = torch.cumsum(inside, 0, dtype=torch.int8)[:total].to(torch.float32)

    def normal(std):
        return torch.randn(total, device="cuda", generator=gen).mul_(inside).mul_(std)

    # gradients: every tensor its own size, and a few elements far above the others
    std = _spread([1e-3 * 4.0 ** (i % 5 - 2) for i in range(len(sizes))], sizes)
    tail = 1 + 20 * (torch.rand(total, device="cuda", generator=gen) < 1e-3)
    g = (normal(1.0) * tail).view(-1, BLOCK).mul_(std).view(-1)
    state = {"case": case, "g": g.to(DTYPE[case["grad"]]), "table": _e8m0("cuda")}
    del tail
    if case["kind"] == "norm":
        state["out"] = torch.zeros(2, device="cuda")
        slices = lambda name: [state[name][f:f + s] for f, s in zip(first, sizes)]  # noqa: E731
        if own:
            from paper_2106_10796_amd import binding
            state["call"] = binding.GradNorm(slices("g"))
        return state
    decay = [DECAY if s >= 4096 else 0.0 for s in sizes]
    state |= {"w": normal(0.05), "t": 100, "out": torch.zeros(2, device="cuda"), "decay": _spread(decay, sizes),
              "first": first, "seed": int(torch.randint(1 << 30, (1,), device="cuda", generator=gen))}
    m = g.mul(0.3).add_((normal(0.2).view(-1, BLOCK) * std).view(-1))
    v = (torch.rand(total, device="cuda", generator=gen) * 2 + 0.1).mul_(inside).view(-1, BLOCK).mul(std * std).view(-1)
    if case["bits"] == 32:
        state |= {"m": m, "v": v}
    else:
        half = torch.full((), 32768, dtype=torch.int32, device="cuda")
        state["m"], state["m_scale"] = _to_8_bits(m, TOP_M, half, state["table"])
        state["v"], state["v_scale"] = _to_8_bits(v, TOP_V, half, state["table"])
        state["m_out"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        state["v_out"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    if case["copy"]:
        state["copy"] = torch.zeros(total, dtype=DTYPE[case["grad"]], device="cuda")
    if own:
        from paper_2106_10796_amd import binding
        tensors, m_out, v_out = [], [], []
        for f, s, d in zip(first, sizes, decay):
            t = {"weight": state["w"][f:f + s], "grad": state["g"][f:f + s], "m": state["m"][f:f + s], "v": state["v"][f:f + s],
                 "weight_decay": d}
            if case["bits"] == 8:
                b = slice(f // BLOCK, (f + s + BLOCK - 1) // BLOCK)
                t |= {"m_scale": state["m_scale"][b], "v_scale": state["v_scale"][b]}
                m_out.append(state["m_out"][f:f + s])
                v_out.append(state["v_out"][f:f + s])
            if case["copy"]:
                t["weight16"] = state["copy"][f:f + s]
            tensors.append(t)
        state["plan"] = binding.AdamWPlan(tensors, grad_dtype=DTYPE[case["grad"]], state_bits=case["bits"])
        if case["bits"] == 8:
            state["plan"].bind_readout(m_out, v_out)
    return state


def _held(rows, cols):
    """Room for a matrix in MXFP4: (codes, scales)."""
    g = _groups(cols)
    return (torch.zeros(rows, 64 * g, dtype=torch.uint8, device="cuda"), torch.zeros(g, rows, 4, dtype=torch.uint8, device="cuda"))


def _prepare_matrix(case, gen):
    m, n, k = case["m"], case["n"], case["k"]
    normal = lambda r, c, s: torch.randn(r, c, device="cuda", generator=gen).mul_(s)  # noqa: E731

    def activations(rows, cols):
        # some channels far larger than the others, as activations have them
        channel = 1 + 15 * (torch.rand(cols, device="cuda", generator=gen) < 0.01)
        return normal(rows, cols, 1.0).mul_(channel)

    state = {"case": case, "table": _e8m0("cuda"), "fp4": torch.tensor(FP4 + tuple(-v for v in FP4), device="cuda")}
    names = {}
    if case["kind"] == "quantize":
        x = normal(m, n, 0.02) if case["x"] == "f32" else activations(m, n)
        state["x"] = x.to(DTYPE[case["x"]])
        if case["row"]:
            names["row"], state["row_out"] = (m, n), torch.zeros(m, n, dtype=DTYPE[case["x"]], device="cuda")
        if case["col"]:
            names["col"], state["col_out"] = (n, m), torch.zeros(n, m, dtype=DTYPE[case["x"]], device="cuda")
        for name, shape in names.items():
            state[name] = _held(*shape)
    elif case["kind"] == "product":
        names = {"a": (m, k), "b": (n, k)}
        state["a"] = _to_mxfp4(activations(m, k), state["table"])
        state["b"] = _to_mxfp4(normal(n, k, k ** -0.5), state["table"])
        state["y"] = torch.zeros(m, n, dtype=DTYPE[case["out"]], device="cuda")
    else:
        w = normal(n, k, k ** -0.5)
        names = {"w": (n, k), "x4": (m, k)}
        state["w"], state["x4"] = _to_mxfp4(w, state["table"]), _held(m, k)
        state["x"] = activations(m, k).to(DTYPE[case["x"]])
        state["y"] = torch.zeros(m, n, dtype=DTYPE[case["x"]], device="cuda")
        if case["train"]:
            names |= {"w_t": (k, n), "x4_t": (k, m), "dy4": (m, n), "dy4_t": (n, m)}
            state["w_t"] = _to_mxfp4(w.t().contiguous(), state["table"])
            state |= {"x4_t": _held(k, m), "dy4": _held(m, n), "dy4_t": _held(n, m)}
            state["dy"] = normal(m, n, 1e-3).to(DTYPE[case["x"]])
            state["dx"] = torch.zeros(m, k, dtype=DTYPE[case["x"]], device="cuda")
            state["dw"] = torch.zeros(n, k, device="cuda")
    if own:
        from paper_2106_10796_amd import binding
        state["own"] = {name: binding.Mxfp4(*state[name], *shape) for name, shape in names.items()}
        if case["kind"] in ("product", "linear"):
            state["work"] = binding.new_mxfp4_workspace([(m, n, k)] + ([(m, k, n), (n, k, m)] if case["train"] else []))
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)
    return _prepare_list(case, gen) if case["kind"] in ("adamw", "norm") else _prepare_matrix(case, gen)


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _mix_seed(seed):
    """32 bits of the call's 64-bit seed."""
    x = (seed + 0x9E3779B97F4A7C15) & (2 ** 64 - 1)
    x = ((x ^ (x >> 32)) * 0xD6E8FEB86659FD93) & (2 ** 64 - 1)
    x ^= x >> 32
    return x & 0xFFFFFFFF


def _signed(x):
    return x - (1 << 32) if x >= 1 << 31 else x


def _hash(n, seed, device):
    """32 bits for each element of the list, as int32."""
    x = torch.arange(n, dtype=torch.int32, device=device) * _signed(0x9E3779B9) + _signed(_mix_seed(seed))
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _signed(0xBB67AE85)
    x = (x ^ ((x >> 13) & 0x7FFFF)) * _signed(0x6A09E667)
    return x ^ ((x >> 16) & 0xFFFF)


def _to_8_bits(x, top, dither, table):
    """Codes and scale bytes of a state; `dither` has 16 bits for each element."""
    b = (x.view(-1, BLOCK).abs().amax(1).view(torch.int32) >> 23) & 0xFF
    # |x| 2^(top - b), in two factors that are powers of two themselves
    up = table[(254 - b).clamp(min=0)][:, None]
    y = x.view(-1, BLOCK).abs().mul(up).mul(2.0 ** (top - 127)).view(-1)
    code = (y.view(torch.int32) + dither.view(-1) * 16) >> 20
    if top == TOP_M:
        code = torch.where(x < 0, code | 128, code)
    else:
        code = torch.where((x > 0) & (code == 0), 1, code)
    return code.to(torch.uint8), b.to(torch.uint8)


def _from_8_bits(codes, scale, top, table):
    c = codes.to(torch.int32)
    mag = ((c & 0x7F if top == TOP_M else c) << 20).view(torch.float32)
    x = mag.mul(2.0 ** (127 - top)).view(-1, BLOCK).mul(table[scale.long()][:, None]).view(-1)
    return torch.where(c > 127, -x, x) if top == TOP_M else x


def _plain_norm(state, scale=1.0):
    norm = (state["g"].float() * scale).square().sum().sqrt()
    state["out"][0] = norm
    state["out"][1] = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
    return state["out"]


def _plain_adamw(state):
    case, t = state["case"], state["t"]
    g = state["g"].float()
    if case["clip"]:
        g = g * _plain_norm(state)[1]
    if case["bits"] == 32:
        m, v = state["m"], state["v"]
    else:
        m = _from_8_bits(state["m"], state["m_scale"], TOP_M, state["table"])
        v = _from_8_bits(state["v"], state["v_scale"], TOP_V, state["table"])
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    denom = v.sqrt() * (1 / (1 - BETA2 ** t) ** 0.5) + EPS
    w = state["w"].view(-1, BLOCK) * (1 - LR * state["decay"])
    state["w"].copy_(w.view(-1) - (m / denom) * (LR / (1 - BETA1 ** t)))
    outs = {"w": state["w"]}
    if case["copy"]:
        outs["copy"] = state["copy"].copy_(state["w"])
    if case["clip"]:
        outs["norm"] = state["out"]
    if case["bits"] == 32:
        state["m"].copy_(m)
        state["v"].copy_(v)
        return outs | {"m": state["m"], "v": state["v"]}
    h = _hash(m.numel(), state["seed"] + t, m.device)
    for name, x, top, dither in (("m", m, TOP_M, h & 0xFFFF), ("v", v, TOP_V, (h >> 16) & 0xFFFF)):
        codes, scale = _to_8_bits(x, top, dither, state["table"])
        state[name].copy_(codes)
        state[name + "_scale"].copy_(scale)
        outs[name] = state[name + "_out"].copy_(_from_8_bits(codes, scale, top, state["table"]))
    return outs


def _to_mxfp4(x, table):
    """(codes, scales) of a matrix in blocks along its rows."""
    rows, cols = x.shape
    g = _groups(cols)
    x = torch.nn.functional.pad(x.float(), (0, 128 * g - cols)).view(rows, 4 * g, 32)
    field = (x.abs().amax(2).view(torch.int32) >> 23) & 0xFF
    s = torch.where(field == 255, 255, (field - 2).clamp(min=0))
    y = x.abs() * table[(254 - s).clamp(min=0)][:, :, None]
    code = (y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    code = (code + 8 * torch.signbit(x)).view(rows, 64 * g, 2)
    return code[:, :, 0] + 16 * code[:, :, 1], s.to(torch.uint8).view(rows, g, 4).transpose(0, 1).contiguous()


def _from_mxfp4(q, rows, cols, state):
    codes, scales = q
    v = state["fp4"][torch.stack((codes & 15, codes >> 4), 2).view(rows, -1, 32).long()]
    s = state["table"][scales.transpose(0, 1).reshape(rows, -1).long()]
    return (v * s[:, :, None]).view(rows, -1)[:, :cols]


def _keep(to, q):
    to[0].copy_(q[0])
    to[1].copy_(q[1])
    return to


def _plain_matrix(state):
    case = state["case"]
    m, n, k = case["m"], case["n"], case["k"]
    held = lambda name, x: _keep(state[name], _to_mxfp4(x, state["table"]))  # noqa: E731
    if case["kind"] == "quantize":
        outs = {}
        if case["row"]:
            outs["row"] = state["row_out"].copy_(_from_mxfp4(held("row", state["x"]), m, n, state))
        if case["col"]:
            outs["col"] = state["col_out"].copy_(_from_mxfp4(held("col", state["x"].t()), n, m, state))
        return outs
    if case["kind"] == "product":
        return {"y": state["y"].copy_(_from_mxfp4(state["a"], m, k, state) @ _from_mxfp4(state["b"], n, k, state).t())}
    x4 = _from_mxfp4(held("x4", state["x"]), m, k, state)
    outs = {"y": state["y"].copy_(x4 @ _from_mxfp4(state["w"], n, k, state).t())}
    if case["train"]:
        x4_t = _from_mxfp4(held("x4_t", state["x"].t()), k, m, state)
        dy4 = _from_mxfp4(held("dy4", state["dy"]), m, n, state)
        dy4_t = _from_mxfp4(held("dy4_t", state["dy"].t()), n, m, state)
        outs["dx"] = state["dx"].copy_(dy4 @ _from_mxfp4(state["w_t"], k, n, state).t())
        outs["dw"] = state["dw"].copy_(dy4_t @ x4_t.t())
    return outs


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------
def _own_list(state):
    case = state["case"]
    if case["kind"] == "norm":
        state["call"].compute(state["out"], max_norm=MAX_NORM)
        return state["out"]
    plan, outs = state["plan"], {"w": state["w"], "m": state["m"], "v": state["v"]}
    if case["clip"]:
        plan.grad_norm(state["out"], max_norm=MAX_NORM)
        outs["norm"] = state["out"]
    plan.step(state["t"], LR, BETA1, BETA2, EPS, seed=state["seed"] + state["t"], clip=state["out"] if case["clip"] else None)
    if case["copy"]:
        outs["copy"] = state["copy"]
    if case["bits"] == 8:
        plan.read_states()
        outs |= {"m": state["m_out"], "v": state["v_out"]}
    return outs


def _own_matrix(state):
    from paper_2106_10796_amd import binding as B
    case, q = state["case"], state["own"]
    if case["kind"] == "quantize":
        B.cdsgd_mxfp4_quantize(state["x"], q.get("row"), q.get("col"))
        outs = {}
        for name in q:
            B.cdsgd_mxfp4_dequantize(q[name], state[name + "_out"])
            outs[name] = state[name + "_out"]
        return outs
    if case["kind"] == "product":
        B.cdsgd_mxfp4_matmul(q["a"], q["b"], state["y"], state["work"])
        return {"y": state["y"]}
    outs = {"y": state["y"]}
    B.cdsgd_mxfp4_quantize(state["x"], q["x4"], q.get("x4_t"))
    B.cdsgd_mxfp4_matmul(q["x4"], q["w"], state["y"], state["work"])
    if case["train"]:
        B.cdsgd_mxfp4_quantize(state["dy"], q["dy4"], q["dy4_t"])
        B.cdsgd_mxfp4_matmul(q["dy4"], q["w_t"], state["dx"], state["work"])
        B.cdsgd_mxfp4_matmul(q["dy4_t"], q["x4_t"], state["dw"], state["work"])
        outs |= {"dx": state["dx"], "dw": state["dw"]}
    return outs


def run(state):
    lists = state["case"]["kind"] in ("adamw", "norm")
    if own:
        outs = _own_list(state) if lists else _own_matrix(state)
    elif state["case"]["kind"] == "norm":
        outs = _plain_norm(state)
    else:
        outs = _plain_adamw(state) if lists else _plain_matrix(state)
    if "t" in state:
        state["t"] += 1
    return outs


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _exact_round_state(x, top, bits16):
    """What an 8-bit state holds after x, from the numbers alone: the grid of a block is that of a float with 3 mantissa
    bits whose largest binade is the one of the block's largest magnitude and which has top - 1 binades below it."""
    mag = x.view(-1, BLOCK).abs()
    # the binade of the largest magnitude as a 32-bit float (denormal ones count as the lowest)
    largest = torch.floor(torch.log2(mag.amax(1, keepdim=True).clamp(min=2.0 ** -126)))
    largest = torch.where(mag.amax(1, keepdim=True) < 2.0 ** -126, -127.0, largest)
    lowest = largest - (top - 1)
    binade = torch.floor(torch.log2(mag.clamp(min=1e-300)))
    step = torch.exp2(torch.maximum(binade, lowest) - 3)
    held = torch.floor(mag / step + bits16.view(-1, BLOCK).double() / 65536) * step
    if top == TOP_V:
        held = torch.where((mag > 0) & (held == 0), step, held)
    return (held * x.view(-1, BLOCK).sign()).view(-1)


def _exact_held_state(codes, scale, top):
    c = codes.to(torch.int64)
    sign, c = (1 - 2 * (c >> 7), c & 127) if top == TOP_M else (torch.ones_like(c), c)
    e, mant = (c >> 3).double(), (c & 7).double()
    value = torch.where(e > 0, torch.exp2(e) * (1 + mant / 8), 2 * mant / 8)          # in units of 2^-127 before the block's scale
    return sign * (value.view(-1, BLOCK) * torch.exp2(scale.double()[:, None] - top - 127)).view(-1)


def _exact_bits(n, seed):
    x = torch.arange(n, dtype=torch.int64, device="cuda") & 0xFFFFFFFF
    low = 0xFFFFFFFF
    z = (seed + 0x9E3779B97F4A7C15) % 2 ** 64
    z = (z ^ (z // 2 ** 32)) * 0xD6E8FEB86659FD93 % 2 ** 64
    x = (x * 0x9E3779B9 + (z ^ (z // 2 ** 32)) % 2 ** 32) & low
    for shift, factor in ((15, 0xBB67AE85), (13, 0x6A09E667)):
        x ^= x // 2 ** shift
        # the low 32 bits of a product of two 32-bit numbers, by halves
        x = ((x & 0xFFFF) * factor + (((x >> 16) * (factor & 0xFFFF) & 0xFFFF) << 16)) & low
    return x ^ (x // 65536)


def _exact_list(case, seed):
    s = prepare(case, seed)
    g = s["g"].double()
    norm = torch.sqrt(torch.sum(g ** 2))
    factor = torch.clamp(MAX_NORM / norm, max=1.0)
    both = torch.stack((norm, factor))
    if case["kind"] == "norm":
        return both
    if case["clip"]:
        g = g * factor
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m, v = _exact_held_state(s["m"], s["m_scale"], TOP_M), _exact_held_state(s["v"], s["v_scale"], TOP_V)
    t = s["t"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    update = (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    w = s["w"].double()
    w = w - LR * (torch.repeat_interleave(s["decay"].double().view(-1), BLOCK) * w + update)
    if case["bits"] == 8:
        h = _exact_bits(m.numel(), s["seed"] + t)
        m, v = _exact_round_state(m, TOP_M, h & 0xFFFF), _exact_round_state(v, TOP_V, h >> 16)
    outs = {"w": w, "m": m, "v": v}
    if case["clip"]:
        outs["norm"] = both
    if case["copy"]:
        outs["copy"] = w
    return outs


def _exact_mxfp4(x):
    """The values that a matrix has after quantisation in blocks along its rows."""
    rows, cols = x.shape
    pad = -cols % 32
    x = torch.cat((x.double(), torch.zeros(rows, pad, dtype=torch.float64, device=x.device)), 1).view(rows, -1, 32)
    scale = torch.exp2(torch.floor(torch.log2(x.abs().amax(2, keepdim=True).clamp(min=2.0 ** -125))) - 2)
    grid = torch.tensor(FP4, dtype=torch.float64, device=x.device)
    y = (x.abs() / scale).clamp(max=6.0)
    upper = torch.searchsorted(grid, y).clamp(1, 7)           # y lies between two neighbours of the grid
    below, above = y - grid[upper - 1], grid[upper] - y
    take = torch.where((above < below) | ((above == below) & (upper % 2 == 0)), upper, upper - 1)
    return (grid[take] * torch.sign(x) * scale).view(rows, -1)[:, :cols]


def _exact_values(q, rows, cols):
    codes, scales = q
    nibbles = torch.empty(rows, 2 * codes.shape[1], dtype=torch.int64, device=codes.device)
    nibbles[:, 0::2], nibbles[:, 1::2] = codes % 16, codes // 16
    e, mant = (nibbles % 8) // 2, (nibbles % 2).double()
    value = torch.where(e > 0, (1 + mant / 2) * torch.exp2(e.double() - 1), mant / 2) * (1 - 2 * (nibbles // 8))
    s = torch.repeat_interleave(scales.permute(1, 0, 2).reshape(rows, -1).double(), 32, 1)
    return (value * torch.exp2(s - 127))[:, :cols]


def _exact_matrix(case, seed):
    s = prepare(case, seed)
    m, n, k = case["m"], case["n"], case["k"]
    if case["kind"] == "quantize":
        outs = {}
        if case["row"]:
            outs["row"] = _exact_mxfp4(s["x"])
        if case["col"]:
            outs["col"] = _exact_mxfp4(s["x"].t().contiguous())
        return outs
    if case["kind"] == "product":
        return {"y": torch.mm(_exact_values(s["a"], m, k), _exact_values(s["b"], n, k).t().contiguous())}
    outs = {"y": torch.mm(_exact_mxfp4(s["x"]), _exact_values(s["w"], n, k).t().contiguous())}
    if case["train"]:
        outs["dx"] = torch.mm(_exact_mxfp4(s["dy"]), _exact_values(s["w_t"], k, n).t().contiguous())
        outs["dw"] = torch.mm(_exact_mxfp4(s["dy"].t().contiguous()), _exact_mxfp4(s["x"].t().contiguous()).t().contiguous())
    return outs


def exact(case, seed):
    return _exact_list(case, seed) if case["kind"] in ("adamw", "norm") else _exact_matrix(case, seed)
