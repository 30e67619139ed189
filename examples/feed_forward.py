"""A feed-forward block with the framework's operators: its program, a few training steps, one token.

    out = x + D2 (D1 gelu(x w1 + b1) w2 + b2)

The program is what the framework's table says about the block's first half as a Spec (Matmul, bias add, ReLU) of the
paper's machine; Table.apply computes the same Spec on data.  Training and decoding run on binding.linear and
binding.linear_grad alone: no mask of either dropout is stored, the gradient draws it again from seed and step.
Normed is the block behind a layer normalisation, Served that with its weights in 4-bit blocks.

    python examples/feed_forward.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_01637_amd import binding as B        # noqa: E402
from paper_2505_01637_amd import workloads as W      # noqa: E402


class FeedForward:
    """Weights in bf16 with f32 master copies; rows of x are tokens."""

    def __init__(self, width, hidden, dropout, seed, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        make = lambda *s: torch.randn(s, generator=gen, device=device) * s[0] ** -0.5
        self.master = [make(width, hidden), torch.zeros(hidden, device=device), make(hidden, width), torch.zeros(width, device=device)]
        self.dropout, self.seed = dropout, seed
        self._round()

    def _round(self):
        self.w1, self.b1, self.w2, self.b2 = (p.bfloat16() for p in self.master)

    def forward(self, x, step=None):
        """step: None without dropout (decoding), else the training step, from which both masks are drawn."""
        p = 0.0 if step is None else self.dropout
        one, two = ({"dropout": p, "seed": self.seed, "offset": 0 if step is None else 2 * step + i} for i in range(2))
        h, z = B.linear(x, self.w1, self.b1, activation="gelu", pre=True, **one)
        out = B.linear(h, self.w2, self.b2, x, **two)
        return out, (x, h, z, one, two)

    def backward(self, grad, saved):
        """(gradient by x, gradients of the four parameters)."""
        x, h, z, one, two = saved
        d_h, d_w2, d_b2 = B.linear_grad(grad, h, self.w2, self.b2, **two)
        d_x, d_w1, d_b1 = B.linear_grad(d_h, x, self.w1, self.b1, z, activation="gelu", **one)
        return d_x + grad, [d_w1, d_b1, d_w2, d_b2]         # (the residual passes grad on)

    def update(self, grads, rate):
        for p, g in zip(self.master, grads):
            p.add_(g.float(), alpha=-rate)
        self._round()

    def token(self, x):
        """One row, no dropout."""
        h = B.linear(x, self.w1, self.b1, activation="gelu")
        return B.linear(h, self.w2, self.b2, x)


class Normed:
    """x + the block's branch of layer_norm(x); scale and shift of the normalisation in f32."""

    def __init__(self, block, device="cuda"):
        width = block.w1.shape[0]
        self.block, self.scale, self.shift = block, torch.ones(width, device=device), torch.zeros(width, device=device)

    def forward(self, x):
        y, stats = B.layer_norm(x, self.scale, self.shift, stats=True)
        b = self.block
        h, z = B.linear(y, b.w1, b.b1, activation="gelu", pre=True)
        return B.linear(h, b.w2, b.b2, x), (x, stats, y, h, z)

    def backward(self, grad, saved):
        """(gradient by x, gradients by scale, shift and the block's four parameters)."""
        x, stats, y, h, z = saved
        b = self.block
        d_h, d_w2, d_b2 = B.linear_grad(grad, h, b.w2, b.b2)
        d_y, d_w1, d_b1 = B.linear_grad(d_h, y, b.w1, b.b1, z, activation="gelu")
        d_x, d_scale, d_shift = B.layer_norm_grad(d_y, x, stats, self.scale, self.shift, grad)
        return d_x, [d_scale, d_shift, d_w1, d_b1, d_w2, d_b2]


class Served:
    """Normed for decoding, its two weight matrices in microscaled 4-bit floating point: a quarter of what bf16 reads."""

    def __init__(self, normed):
        self.normed = normed
        self.w1, self.w2 = (B.mx_quantize(w, dim=-2) for w in (normed.block.w1, normed.block.w2))

    def token(self, x):
        n = self.normed
        h = B.mx_linear(B.layer_norm(x, n.scale, n.shift), self.w1, n.block.b1, activation="gelu")
        return B.mx_linear(h, self.w2, n.block.b2, x)


def program(width, hidden, rows):
    """The program of relu(x w1 + b1), rows x width by width x hidden in f32, and the Spec computed on data."""
    cfg = W.config(5, max_size=max(width, hidden, rows))
    target, tables = B.solve_config(cfg)
    fused = tables["F"]
    top = cfg["target"]["n_levels"] - 1
    x = fused.coord_of_spec((1, rows, width, hidden), [top] * 5, layouts=[0] * 4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lhs, rhs, bias = (torch.randn(s, generator=gen, device="cuda") for s in ((rows, width), (width, hidden), (hidden,)))
    return fused.program_text(x), fused.apply(x, lhs, rhs, bias), torch.relu(lhs @ rhs + bias)


def train(steps=60, width=256, hidden=1024, rows=512, rate=0.02, dropout=0.1):
    """Losses of a regression on a fixed batch."""
    model = FeedForward(width, hidden, dropout, seed=7)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    want = torch.roll(x.float(), 1, dims=1)
    losses = []
    for step in range(steps):
        out, saved = model.forward(x, step)
        diff = out.float() - want
        losses.append(diff.square().mean().item())
        _, grads = model.backward((2.0 / rows * diff).bfloat16(), saved)
        model.update(grads, rate)
    return model, losses


if __name__ == "__main__":
    text, got, want = program(16, 32, 8)
    print(text)
    print("the Spec on data, largest difference from torch: %.2g" % (got - want).abs().max().item())
    model, losses = train()
    print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], len(losses)))
    x = torch.randn(1, 256, device="cuda").bfloat16()
    print("one token:", tuple(model.token(x).shape))
    normed = Normed(model)
    served, whole = Served(normed).token(x).float(), normed.forward(x)[0].float()
    print("behind a normalisation, weights in 4 bits: %.2g of its norm from bf16" % ((served - whole).norm() / whole.norm()).item())
