"""The feed-forward example: the Spec that its table names, its training steps, a token."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_feed_forward_example():
    import torch
    import feed_forward as F
    text, got, want = F.program(16, 32, 8)
    assert "bufferize" in text or "microkernel" in text
    # sums of 16 products in f32, both sides: 18 units each of sums of magnitudes below 16 * 25
    assert (got - want).abs().max().item() < 36 * 2.0 ** -24 * 400
    model, losses = F.train()
    assert all(l == l for l in losses) and losses[-1] < 0.5 * losses[0]
    x = torch.randn(3, 256, device="cuda").bfloat16()
    rows, _ = model.forward(x)
    alone = torch.cat([model.token(x[i:i + 1]) for i in range(3)])
    # the same formula, its sums in another order: one rounding unit of bf16 of h and of out
    assert (rows.float() - alone.float()).abs().max().item() <= 2.0 ** -7 * rows.float().abs().max().item()


@pytest.mark.gpu
def test_feed_forward_gradient_is_that_of_its_parts():
    """backward against autograd of the formula in f64 with the example's own masks (from ones through binding.dropout)."""
    import torch
    import feed_forward as F
    from paper_2505_01637_amd import binding as B
    model = F.FeedForward(64, 96, 0.2, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(40, 64, generator=gen, device="cuda").bfloat16()
    out, saved = model.forward(x, step=5)
    g = torch.randn(40, 64, generator=gen, device="cuda").bfloat16()
    d_x, grads = model.backward(g, saved)
    masks = [B.dropout(torch.ones(40, n, device="cuda"), dropout=0.2, seed=3, offset=10 + i).double() for i, n in enumerate((96, 64))]
    ps = [p.double().requires_grad_() for p in (x, model.w1, model.b1, model.w2, model.b2)]
    h = torch.nn.functional.gelu(ps[0] @ ps[1] + ps[2], approximate="tanh") * masks[0]
    want = ps[0] + (h @ ps[3] + ps[4]) * masks[1]
    want.backward(g.double())
    # chained bf16 roundings (z, h, out, d_h, dz, the gradients): ten units of 2^-8, of the norm, as they are independent
    for got, p in zip([d_x] + grads, ps):
        assert (got.double() - p.grad).norm().item() <= 10 * 2.0 ** -8 * p.grad.norm().item()
    assert (out.double() - want).norm().item() <= 4 * 2.0 ** -8 * want.norm().item()
