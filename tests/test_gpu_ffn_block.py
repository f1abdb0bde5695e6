"""The three calls of a feed-forward block together: units handed from call to call, a prompt against its tokens one by
one, the gradient of the whole, and the example that runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("ffn_block", os.path.join(ROOT, "examples", "ffn_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def decoded(hif4, units):
    return hif4.hif4_dequantize(units, torch.float32).double()


@pytest.mark.parametrize("tokens,hidden,inner", [(1, 256, 512), (8, 512, 1024), (40, 512, 1088), (200, 768, 1024)])
def test_block_against_the_formula(example, tokens, hidden, inner):
    """From the units that each call wrote: the next call's result within the product's tolerance (1e-5 sum |a||b|), the
    activation's 2^-18 and one rounding to BF16."""
    import paper_2602_11287_b200 as hif4
    block = example.FeedForward(hidden, inner, seed=3)
    x = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    r = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    w = (1 + 0.1 * torch.randn(hidden, device="cuda")).to(torch.bfloat16)
    h, y, out = block.forward(x, r, w)
    f = hif4.hif4_gated_linear(y, block.gate, block.up, dtype=torch.bfloat16, units=True)
    Y, G, U, F, D = (decoded(hif4, t) for t in (y, block.gate, block.up, f, block.down))
    rows = hif4.hif4_gated_linear(y, block.gate, block.up, dtype=torch.bfloat16)
    assert torch.equal(f, hif4.hif4_quantize(rows))
    g, u = Y @ G.t(), Y @ U.t()
    eg, eu = 1e-5 * (Y.abs() @ G.abs().t()), 1e-5 * (Y.abs() @ U.abs().t())
    a = g * torch.sigmoid(g)
    bound = 2.0 ** -8 * (a * u).abs() + (1.2 * eg + 2.0 ** -18 * a.abs()) * (u.abs() + eu) + a.abs() * eu
    assert ((rows.double() - a * u).abs() <= bound).all()
    want = F @ D.t() + h.double()
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * (F.abs() @ D.abs().t()) + 2.0 ** -18 * h.double().abs()).all()


def test_a_prompt_and_its_tokens_one_by_one(example):
    """Rows of a block are independent: streaming form (one token) and tensor-core form (the prompt) differ by the order of
    FP32 sums only, so by roundings at the edge: the norm of the difference stays within 2^-7 of the result's."""
    block = example.FeedForward(512, 1024, seed=5)
    x = torch.randn(64, 512, device="cuda").to(torch.bfloat16)
    w = torch.ones(512, device="cuda", dtype=torch.bfloat16)
    zero = torch.zeros_like(x)
    together = block(x, zero, w).double()
    alone = torch.cat([block(x[i:i + 1], zero[i:i + 1], w) for i in range(64)]).double()
    assert float((together - alone).norm() / together.norm()) <= 2.0 ** -7


def test_gradient_of_the_block_points_downhill(example):
    """The loss falls over a few steps, and a small step along the gradient changes it by about its squared norm: the step is
    sized to change h by a tenth of its size, where conversion noise (2^-4 of an element, averaged over 128 x 256) is small."""
    losses = example.fit_prompt(hidden=256, inner=512, tokens=128, steps=40)
    assert losses[-1] < 0.5 * losses[0]


def test_example_runs(example, capsys):
    losses = example.main(["--hidden", "256", "--inner", "512", "--tokens", "64", "--steps", "8"])
    assert losses[-1] < losses[0]
    assert "soft prompt" in capsys.readouterr().out
