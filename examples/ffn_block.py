"""A transformer block's feed-forward half on frozen HiF4 weights: serving it, and training what lies around the weights.

    python examples/ffn_block.py [--hidden 1024] [--inner 4096] [--tokens 256] [--steps 30]

Three calls run the block: the norm with its residual writes HiF4 units, the gated projections read them and write units,
the down projection reads those and adds the residual.  Their gradient calls reach the norm weight and whatever produced
the block's input; here a soft prompt is fitted so that the block's output matches a target.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_11287_b200 as hif4  # noqa: E402


class FeedForward:
    """out = h + W_down HiF4(silu(W_gate y) * W_up y) with h = residual + x and y = HiF4(rms_norm(h) * weight)."""

    def __init__(self, hidden: int, inner: int, seed: int = 0, eps: float = 1e-5):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def units(rows, cols):
            w = torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5
            return hif4.hif4_quantize(w.to(torch.bfloat16))

        self.gate, self.up, self.down = units(inner, hidden), units(inner, hidden), units(hidden, inner)
        self.eps = eps

    def __call__(self, x, residual, weight):
        return _Block.apply(x, residual, weight, self)

    def forward(self, x, residual, weight):
        h, y = hif4.hif4_block_norm(x, weight, residual=residual, eps=self.eps, units=True)
        f = hif4.hif4_gated_linear(y, self.gate, self.up, act=hif4.HIF4_ACT_SILU, dtype=x.dtype, units=True)
        return h, y, hif4.hif4_linear_act(f, self.down, residual=h, dtype=x.dtype)

    def backward(self, dout, h, y, weight):
        df, _ = hif4.hif4_linear_act_backward(dout, None, self.down)
        dy, _, _ = hif4.hif4_gated_linear_backward(df, y, self.gate, self.up, act=hif4.HIF4_ACT_SILU)
        return hif4.hif4_block_norm_backward(dy, h, weight, dh=dout, eps=self.eps)


class _Block(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, block):
        h, y, out = block.forward(x, residual, weight)
        ctx.block = block
        ctx.save_for_backward(h, y, weight)
        return out

    @staticmethod
    def backward(ctx, dout):
        h, y, weight = ctx.saved_tensors
        d = ctx.block.backward(dout.contiguous(), h, y, weight)
        return d["dx"], d["dresidual"], d["dweight"].to(weight.dtype), None


def fit_prompt(hidden: int, inner: int, tokens: int, steps: int, rate: float = 0.5):
    """Losses of a soft prompt that is fitted through the frozen block."""
    block = FeedForward(hidden, inner)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    residual = torch.randn(tokens, hidden, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn(tokens, hidden, generator=g, device="cuda").to(torch.bfloat16)
    prompt = torch.zeros(tokens, hidden, device="cuda", requires_grad=True)
    weight = torch.ones(hidden, device="cuda", requires_grad=True)
    optimizer = torch.optim.Adam([prompt, weight], lr=rate / 10)
    losses = []
    for _ in range(steps):
        optimizer.zero_grad()
        out = block(prompt.to(torch.bfloat16), residual, weight.to(torch.bfloat16))
        loss = (out.float() - target.float()).square().mean()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=4096)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args(argv)
    block = FeedForward(a.hidden, a.inner)
    weight = torch.ones(a.hidden, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(a.tokens, a.hidden, device="cuda").to(torch.bfloat16)
    prompt = block(x, torch.zeros_like(x), weight)
    last = block(x[-1:], torch.zeros_like(x[-1:]), weight)
    print(f"prompt of {a.tokens} tokens {tuple(prompt.shape)}; its last token alone differs by "
          f"{float((prompt[-1:].float() - last.float()).abs().max()):.2g}")
    losses = fit_prompt(a.hidden, a.inner, a.tokens, a.steps)
    print(f"loss of the soft prompt {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    return losses


if __name__ == "__main__":
    main()
