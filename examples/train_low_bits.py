"""Two linear layers, held and multiplied in microscaled 4-bit floating point, learn from several workers' 2-bit gradients.

A step: every worker's forward and backward products (cdsgd_mxfp4_quantize, cdsgd_mxfp4_matmul), its gradients to two bits an element
with what is left kept for the next step (cdsgd_quantize_pack), their sum (cdsgd_decode_sum), the sum's norm and AdamW with states in
eight bits (AdamWPlan.grad_norm, AdamWPlan.step), and the new weights back to four bits.  The workers share one GPU here; their packed
gradients are all that would cross a network.  At the end the model answers a single token, and the states are read out
(AdamWPlan.read_states).

    python examples/train_low_bits.py [--steps 200] [--tokens 512] [--width 256] [--hidden 1024] [--workers 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2106_10796_amd as cd  # noqa: E402


class Linear:
    """y = x w^T: the weight in 32 bits for the optimiser, and in 4 bits along its rows (forward) and its columns (backward)."""

    def __init__(self, outs, ins, tokens, workers, gen):
        self.w = torch.randn(outs, ins, device="cuda", generator=gen) * ins ** -0.5
        self.q, self.q_t = cd.new_mxfp4(outs, ins), cd.new_mxfp4(ins, outs)
        self.x, self.x_t = cd.new_mxfp4(tokens, ins), cd.new_mxfp4(ins, tokens)
        self.dy, self.dy_t = cd.new_mxfp4(tokens, outs), cd.new_mxfp4(outs, tokens)
        self.y = torch.empty(tokens, outs, dtype=torch.bfloat16, device="cuda")
        self.dx = torch.empty(tokens, ins, dtype=torch.bfloat16, device="cuda")
        self.dw, self.sum = torch.empty_like(self.w), torch.empty_like(self.w)
        self.left = [torch.zeros_like(self.w) for _ in range(workers)]
        self.packed = [cd.new_packed(self.w.numel()) for _ in range(workers)]
        self.workspace = cd.new_mxfp4_workspace([(tokens, outs, ins), (tokens, ins, outs), (outs, ins, tokens)])
        self.hold()

    def hold(self):
        cd.cdsgd_mxfp4_quantize(self.w, self.q, self.q_t)

    def forward(self, x):
        cd.cdsgd_mxfp4_quantize(x, self.x, self.x_t)
        cd.cdsgd_mxfp4_matmul(self.x, self.q, self.y, self.workspace)
        return self.y

    def backward(self, dy, worker, threshold, need_dx):
        cd.cdsgd_mxfp4_quantize(dy, self.dy, self.dy_t)
        cd.cdsgd_mxfp4_matmul(self.dy_t, self.x_t, self.dw, self.workspace)
        cd.cdsgd_quantize_pack(self.dw, self.left[worker], self.packed[worker], threshold)
        if need_dx:
            cd.cdsgd_mxfp4_matmul(self.dy, self.q_t, self.dx, self.workspace)
        return self.dx

    def answer(self, x):
        """A few tokens that nothing is learnt from."""
        q = cd.new_mxfp4(*x.shape)
        y = torch.empty(x.shape[0], self.w.shape[0], dtype=x.dtype, device="cuda")
        cd.cdsgd_mxfp4_quantize(x, q)
        cd.cdsgd_mxfp4_matmul(q, self.q, y, cd.new_mxfp4_workspace([(x.shape[0], self.w.shape[0], x.shape[1])]))
        return y

    def state(self, decay):
        n = self.w.numel()
        byte = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
        return dict(weight=self.w, grad=self.sum, m=byte(n), v=byte(n), m_scale=byte(cd.state_blocks(n)), v_scale=byte(cd.state_blocks(n)),
                    weight_decay=decay)


def train(steps=200, tokens=512, width=256, hidden=1024, workers=2, lr=1e-3, threshold=3e-3, max_norm=1.0, seed=0):
    """The loss of every step, the answer to one token beside the teacher's, and the layers' first moments.

    The threshold is well above what most elements of a gradient hold: below it, more is left over in each step than one threshold
    an element can send, and what arrives is old."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    teacher = [rnd(hidden, width) * width ** -0.5, rnd(width, hidden) * hidden ** -0.5]
    taught = lambda x: torch.relu(x.float() @ teacher[0].t().contiguous()) @ teacher[1].t().contiguous()  # noqa: E731
    layers = [Linear(hidden, width, tokens, workers, gen), Linear(width, hidden, tokens, workers, gen)]
    plan = cd.AdamWPlan([layer.state(0.01) for layer in layers], state_bits=8)
    moments = [[torch.empty_like(layer.w) for layer in layers] for _ in range(2)]
    plan.bind_readout(*moments)
    clip, losses = torch.empty(2, device="cuda"), torch.zeros(steps, device="cuda")
    for step in range(1, steps + 1):
        for worker in range(workers):
            x = rnd(tokens, width).bfloat16()
            h = torch.relu(layers[0].forward(x))
            off = layers[1].forward(h).float() - taught(x)
            losses[step - 1] += off.square().mean() / workers
            dh = layers[1].backward((off * (2.0 / off.numel())).bfloat16(), worker, threshold, True)
            layers[0].backward(dh * (h > 0), worker, threshold, False)
        for layer in layers:
            cd.cdsgd_decode_sum(layer.packed, layer.sum, threshold)
        plan.grad_norm(clip, grad_scale=1.0 / workers, max_norm=max_norm)
        plan.step(step, lr * min(1.0, step / 10), grad_scale=1.0 / workers, seed=step, clip=clip)
        for layer in layers:
            layer.hold()
    plan.read_states()
    x = rnd(1, width).bfloat16()
    return losses.tolist(), (layers[1].answer(torch.relu(layers[0].answer(x))).float(), taught(x)), moments[0]


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("steps", 200), ("tokens", 512), ("width", 256), ("hidden", 1024), ("workers", 2)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    losses, (said, right), moments = train(a.steps, a.tokens, a.width, a.hidden, a.workers)
    for i in range(0, a.steps, max(a.steps // 10, 1)):
        print("step %4d  loss %.4f" % (i + 1, losses[i]))
    print("step %4d  loss %.4f" % (a.steps, losses[-1]))
    print("one token: off by %.3f of its size" % float((said - right).norm() / right.norm()))
    print("first moments: rms " + ", ".join("%.2e" % float(m.square().mean().sqrt()) for m in moments))


if __name__ == "__main__":
    main()
