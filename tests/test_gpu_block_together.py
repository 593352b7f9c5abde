"""The operators between a block's products as they are used: a whole block with its products in four bits, forward and backward, against the
same block in 64 bits; activations that live in 8 bits from the one pass to the other; and the two ways of marshalling a call."""
import pytest
import torch

from paper_2106_10796_amd import binding as B

pytestmark = pytest.mark.gpu


class Declines:
    """In the place of the native calls: every call declines."""

    def __getattr__(self, name):
        return lambda *a: -1


class Linear:
    """y = x w^T in four bits, and both gradients.  Holds the values that its operands stand for, for the same in 64 bits."""

    def __init__(self, outs, ins, tokens, gen):
        self.shape, self.tokens = (outs, ins), tokens
        self.w = (torch.randn(outs, ins, device="cuda", generator=gen) * ins ** -0.5).bfloat16()
        self.q, self.q_t = B.new_mxfp4(outs, ins), B.new_mxfp4(ins, outs)
        B.cdsgd_mxfp4_quantize(self.w, self.q, self.q_t)
        self.x, self.x_t, self.dy, self.dy_t = (B.new_mxfp4(*s) for s in ((tokens, ins), (ins, tokens), (tokens, outs), (outs, tokens)))
        self.room = B.new_mxfp4_workspace([(tokens, outs, ins), (tokens, ins, outs), (outs, ins, tokens)])
        self.y, self.dx = (torch.empty(tokens, n, dtype=torch.bfloat16, device="cuda") for n in (outs, ins))
        self.dw = torch.empty(outs, ins, device="cuda")

    def forward(self, x):
        B.cdsgd_mxfp4_quantize(x, self.x, self.x_t)
        B.cdsgd_mxfp4_matmul(self.x, self.q, self.y, self.room)
        return self.y

    def backward(self, dy):
        B.cdsgd_mxfp4_quantize(dy, self.dy, self.dy_t)
        B.cdsgd_mxfp4_matmul(self.dy, self.q_t, self.dx, self.room)
        B.cdsgd_mxfp4_matmul(self.dy_t, self.x_t, self.dw, self.room)
        return self.dx

    @staticmethod
    def _values(q):
        out = torch.empty(q.rows, q.cols, device="cuda")
        B.cdsgd_mxfp4_dequantize(q, out)
        return out.double()

    def exact(self):
        """y, dx and dw of the operands that the products took, in 64 bits."""
        v = self._values
        return v(self.x) @ v(self.q).t(), v(self.dy) @ v(self.q_t).t(), v(self.dy_t) @ v(self.x_t).t()


class Block:
    """Norm, attention, norm with gate and residual, gated activation, and the residual of the next block's norm."""

    def __init__(self, lens, width, heads, kv, dim, hidden, seed, eight):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        T = self.tokens = sum(lens)
        self.lens, self.heads, self.kv, self.dim, self.width, self.hidden, self.eight = lens, heads, kv, dim, width, hidden, eight
        self.starts = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        vector = lambda mean: mean + 0.1 * torch.randn(width, device="cuda", generator=gen)  # noqa: E731
        self.norms = [B.BlockNorm(vector(1.0)), B.BlockNorm(vector(1.0), vector(1.0), vector(0.5), scale=0.8), B.BlockNorm(vector(1.0), None, vector(0.5))]
        self.qkv, self.proj = Linear((heads + 2 * kv) * dim, width, T, gen), Linear(width, heads * dim, T, gen)
        self.up, self.down = Linear(2 * hidden, width, T, gen), Linear(width, hidden, T, gen)
        self.h = torch.randn(T, width, device="cuda", generator=gen)
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.ys, self.rstd = [bf(T, width) for _ in range(3)], [torch.empty(2, T, device="cuda") for _ in range(3)]
        self.hs = [self.h] + [torch.empty_like(self.h) for _ in range(2)]
        self.out, self.lse, self.act = bf(T, heads, dim), torch.empty(heads, T, device="cuda"), bf(T, hidden)
        self.room = [B.new_block_norm_workspace(T, width), B.new_attention_workspace(bf(T, heads, dim), bf(T, kv, dim), seqs=len(lens), train=True)]
        self.h8, self.b8 = ([B.new_mxint8(T, width) if eight else None for _ in range(3)] for _ in range(2))
        self.a8, self.u8 = (B.new_mxint8(T, hidden) if eight else None for _ in range(2))
        self.dy = torch.randn(T, width, device="cuda", generator=gen).bfloat16()
        self.dh = [torch.empty_like(self.h) for _ in range(3)]
        self.grads = [[None if t is None else torch.empty_like(t) for t in n._weights] for n in self.norms]
        self.d_qkv, self.d_gate, self.db = bf(T, (heads + 2 * kv) * dim), bf(T, 2 * hidden), [None, bf(T, width), bf(T, width)]

    def split(self, t):
        at = [0, self.heads * self.dim, (self.heads + self.kv) * self.dim, (self.heads + 2 * self.kv) * self.dim]
        return [t[:, a:b].unflatten(1, (-1, self.dim)) for a, b in zip(at, at[1:])]

    def norm(self, i, block=None):
        self.norms[i].forward(self.hs[max(i - 1, 0)], self.ys[i], self.rstd[i], block=block, h_out=self.hs[i] if i else None, h8=self.h8[i],
                              block8=self.b8[i] if i else None)
        return self.ys[i]

    def forward(self):
        q, k, v = self.split(self.qkv.forward(self.norm(0)))
        B.cdsgd_attention_forward(q, k, v, self.out, self.lse, self.starts, workspace=self.room[1])
        x = self.up.forward(self.norm(1, self.proj.forward(self.out.flatten(1))))
        B.cdsgd_gated_forward(x[:, :self.hidden], x[:, self.hidden:], self.act, self.a8, self.u8)
        return self.norm(2, self.down.forward(self.act))

    def norm_back(self, i, dy, dh_out, block):
        self.norms[i].backward(dy, self.h8[i] or self.hs[i], self.rstd[i], self.dh[i], self.grads[i][0], self.room[0], dh_out=dh_out,
                               block=self.b8[i] or block if i else None, dblock=self.db[i], dblock_weight=self.grads[i][1], dgate=self.grads[i][2])
        return self.db[i]

    def backward(self):
        x, half = self.up.y, self.hidden
        d = self.down.backward(self.norm_back(2, self.dy, None, self.down.y))
        B.cdsgd_gated_backward(d, self.a8 or x[:, :half], self.u8 or x[:, half:], self.d_gate[:, :half], self.d_gate[:, half:])
        d = self.proj.backward(self.norm_back(1, self.up.backward(self.d_gate), self.dh[2], self.proj.y)).unflatten(1, (self.heads, self.dim))
        B.cdsgd_attention_backward(d, *self.split(self.qkv.y), self.out, self.lse, *self.split(self.d_qkv), self.starts, workspace=self.room[1])
        self.norm_back(0, self.qkv.backward(self.d_qkv), self.dh[1], None)
        return self.dh[0]

    def results(self):
        return [*self.hs[1:], *self.ys, self.out, self.act, *self.dh, *[t for g in self.grads for t in g if t is not None], self.d_qkv, self.d_gate,
                *[layer.dw for layer in (self.qkv, self.proj, self.up, self.down)]]


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


CASES = [([50, 1, 93], 96, 6, 2, 24, 200), ([300, 212], 256, 4, 4, 64, 512)]


@pytest.mark.parametrize("case", CASES, ids=["odd", "even"])
@pytest.mark.parametrize("eight", [False, True])
def test_a_block_forward_and_backward(case, eight):
    """Every operator of the run against 64 bits at the inputs that it got there.  Results are 16-bit: off by half a step (2^-9) of each on average
    less than 2^-8 all together, P and dS by as much again, which four halves of 2^-8 are more than; the 8-bit forms are decoded, not bounded."""
    b = Block(*case, seed=1, eight=eight)
    b.forward()
    b.backward()
    limit, T = 4 * 2.0 ** -9, b.tokens
    for layer in (b.qkv, b.proj, b.up, b.down):
        for got, want in zip((layer.y, layer.dx, layer.dw), layer.exact()):
            assert off(got, want) < limit
    # attention, by differentiation in 64 bits
    q, k, v = (t.double().requires_grad_() for t in b.split(b.qkv.y))
    outs, first = [], 0
    for n in b.lens:
        rows = slice(first, first + n)
        heads = lambda t: t[rows].transpose(0, 1).repeat_interleave(b.heads // t.shape[1], 0)  # noqa: E731
        s = torch.matmul(heads(q), heads(k).transpose(1, 2).contiguous()) * b.dim ** -0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        outs.append(torch.matmul(torch.softmax(s, 2), heads(v)).transpose(0, 1))
        first += n
    want = torch.cat(outs)
    assert off(b.out, want.detach()) < limit
    dout = b.proj.dx.unflatten(1, (b.heads, b.dim)).double()
    for got, g in zip(b.split(b.d_qkv), torch.autograd.grad(want, (q, k, v), dout)):
        assert off(got, g) < limit
    # the gated activation and the norms, at what the backward pass read
    value = lambda x8, x: x.double() if x8 is None else decoded(x8)  # noqa: E731
    a, u = (value(x8, x).requires_grad_() for x8, x in ((b.a8, b.up.y[:, :b.hidden]), (b.u8, b.up.y[:, b.hidden:])))
    assert off(b.act, torch.nn.functional.silu(b.up.y[:, :b.hidden].double()) * b.up.y[:, b.hidden:].double()) < limit
    for got, g in zip((b.d_gate[:, :b.hidden], b.d_gate[:, b.hidden:]), torch.autograd.grad(torch.nn.functional.silu(a) * u, (a, u), b.down.dx.double())):
        assert off(got, g) < limit
    for i, (dy, dh_out, block) in enumerate(((b.qkv.dx, b.dh[1], None), (b.up.dx, b.dh[2], b.proj.y), (b.dy, None, b.down.y))):
        w, w_b, gate = (None if t is None else t.double() for t in b.norms[i]._weights)
        one = torch.ones(b.width, dtype=torch.float64, device="cuda")
        r = b.rstd[i][0].double()[:, None]
        h = value(b.h8[i], b.hs[i])
        if block is not None:
            n = b.rstd[i][1].double()[:, None] if w_b is not None else 1.0
            into = b.norms[i].scale * (one if gate is None else gate) * (one if w_b is None else w_b)
            assert off(b.hs[i], b.hs[i - 1].double() + into * n * block.double()) < 2.0 ** -20
        assert off(b.ys[i], b.hs[i].double() * r * w) < limit
        g = dy.double() * w
        t = (0 if dh_out is None else dh_out.double()) + r * (g - h * r * (g * h * r).mean(1, keepdim=True))
        assert off(b.dh[i], t) < 2.0 ** -18 and off(b.grads[i][0], (dy.double() * h * r).sum(0)) < 2.0 ** -18
        if block is not None:
            c = value(b.b8[i], block) * n
            e = t * into
            assert off(b.db[i], n * (e - c * (e * c).mean(1, keepdim=True)) if w_b is not None else e) < limit
            if w_b is not None:
                assert off(b.grads[i][1], (t * c * b.norms[i].scale * (one if gate is None else gate)).sum(0)) < 2.0 ** -18
            assert off(b.grads[i][2], (t * c * b.norms[i].scale * (one if w_b is None else w_b)).sum(0)) < 2.0 ** -18
    assert T == b.out.shape[0]


def decoded(q):
    out = torch.empty(q.rows, q.cols, device="cuda")
    B.cdsgd_mxint8_dequantize(q, out)
    return out.double()


@pytest.mark.parametrize("eight", [False, True])
def test_both_ways_of_marshalling_do_the_same(monkeypatch, eight):
    assert type(B._native()).__name__ == "module"
    runs = []
    for native in (True, False):
        b = Block(*CASES[0], seed=3, eight=eight)
        if not native:
            monkeypatch.setattr(B, "_calls", Declines())
        b.forward()
        b.backward()
        if eight:
            B.cdsgd_mxint8_quantize(b.h, b.h8[0])
            B.cdsgd_mxint8_dequantize(b.h8[0], b.hs[2])
        runs.append([t.clone() for t in b.results()])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


def test_a_captured_step_beside_an_eager_one():
    """The block's step captured and replayed between eager steps of another block that shares nothing with it, on two streams."""
    a, b = Block(*CASES[0], seed=5, eight=True), Block(*CASES[0], seed=6, eight=True)
    side = torch.cuda.Stream()
    for block in (a, b):
        block.forward()
        block.backward()
    want = [[t.clone() for t in block.results()] for block in (a, b)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.forward()
        a.backward()
    for _ in range(3):
        for block in (a, b):
            for t in block.results():
                if t is not block.h:
                    t.fill_(2.0)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        for block, results in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip(block.results(), results))
