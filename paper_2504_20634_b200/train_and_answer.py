"""Train a small network with 4-bit weights, then answer with them one token at a time.

    python -m paper_2504_20634_b200.train_and_answer [--steps N] [--state-bits 8|32]

Algorithm 1 carried to 4 bits, with the three operators in the order a program uses them.  Every step rounds the binary32
master weights to 4 bits stochastically (``fbsr_round_w4``) and runs forward and backward on the values that the codes stand
for; one call then updates the masters of all layers (``fbsr_adamw_multi``, moments in 8 bits by default).  After training
the codes themselves answer single tokens (``fbsr_gemv_w4``); nothing is converted in between.  The task is synthetic: the
student learns a fixed random network of its own shape.
"""
import argparse

import torch

from . import binding as fbsr


class FourBitNetwork:
    """Two layers, relu between them; masters in binary32, moments in `state_bits`, weights in 4 bits with bfloat16 scales."""

    def __init__(self, width, hidden, state_bits=8, group=64, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        shapes = ((hidden, width), (width, hidden))
        self.masters = [torch.randn(s, device=device, generator=gen) * s[1] ** -0.5 for s in shapes]
        self.values = [torch.empty_like(w) for w in self.masters]
        self.grads = [torch.zeros_like(w) for w in self.masters]
        self.group, self.seed = group, seed
        self.offsets, at = [], 0                     # places in the stream of draws: whole padded rows, a multiple of 256 apart
        for w in self.masters:
            self.offsets.append(at)
            at += -(-w.shape[0] * fbsr.fbsr_w4_padded(w.shape[1]) // 256) * 256
        if state_bits == 32:
            state = [[torch.zeros_like(w) for w in self.masters] for _ in range(2)]
            scales = {}
        else:
            state = [[torch.zeros(w.shape, dtype=torch.uint8, device=device) for w in self.masters] for _ in range(2)]
            blocks = [-(-w.numel() // fbsr.ADAMW_BLOCK) for w in self.masters]
            scales = {name: [torch.zeros(b, device=device) for b in blocks] for name in ("m_scale", "v_scale")}
        self.tensors = fbsr.FbsrAdamwTensors(self.masters, self.grads, *state, offsets=self.offsets, **scales)
        self.codes = [None] * len(self.masters)

    def round(self, step):
        """The masters in 4 bits, with the draws of this step."""
        for i, w in enumerate(self.masters):
            self.codes[i] = fbsr.fbsr_round_w4(w, "srf", 4, self.seed + step, offset=self.offsets[i], group=self.group,
                                               scale_fmt="bf16", values=self.values[i])

    def step(self, x, target, step, lr=3e-3):
        """One training step; returns the loss."""
        self.round(step)
        a, b = self.values
        h = torch.relu(x @ a.T)
        error = h @ b.T - target
        # backward through the rounded weights, the rounding itself passed straight through
        g = error * (2.0 / error.numel())
        torch.mm(g.T, h, out=self.grads[1])
        torch.mm(((g @ b) * (h > 0)).T, x, out=self.grads[0])
        fbsr.fbsr_adamw_multi(self.tensors, "srf", 4, self.seed + step, lr, 0.9, 0.99, 1e-8, 0.0, step)
        return error.square().mean()

    def answer(self, token):
        """One token (a row of bfloat16) through the codes of the last rounding."""
        h = torch.relu(fbsr.fbsr_gemv_w4(token, *self.codes[0], group=self.group))
        return fbsr.fbsr_gemv_w4(h, *self.codes[1], group=self.group, out_dtype=torch.float32)


def run(steps=300, state_bits=8, width=256, hidden=512, batch=512, seed=1):
    """Returns the first and the last training loss, the loss of the answers given token by token, and the loss of answering
    with zeros."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    teacher = [torch.randn(s, device="cuda", generator=gen) * s[1] ** -0.5 for s in ((hidden, width), (width, hidden))]

    def task(n):
        x = torch.randn(n, width, device="cuda", generator=gen)
        return x, torch.relu(x @ teacher[0].T) @ teacher[1].T

    net = FourBitNetwork(width, hidden, state_bits, seed=seed + 1000)
    losses = []
    for step in range(1, steps + 1):
        losses.append(net.step(*task(batch), step))
    net.round(steps + 1)
    x, target = task(64)
    answers = torch.stack([net.answer(token) for token in x.to(torch.bfloat16)])
    return float(losses[0]), float(losses[-1]), float((answers - target).square().mean()), float(target.square().mean())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = p.parse_args()
    first, last, answered, zero = run(a.steps, a.state_bits)
    print("loss %.4f -> %.4f in %d steps; answered token by token %.4f (zeros: %.4f)" % (first, last, a.steps, answered, zero))
