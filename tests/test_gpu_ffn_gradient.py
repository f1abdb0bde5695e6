"""The gradient of the whole feed-forward block against the formula in 64 bits on the decoded operands, straight through the
conversions.

Tolerances, in the order of the chain.  dF is one product (1e-5 of the sum of |a||b|) and one rounding to BF16 (2^-8); dG and dU carry
dF's error, the products' and the activation's (slopes of at most 1.2 and 2, 2^-18 of the value) and are rounded to BF16 on the
way into the next product; dY carries theirs through |W| and is rounded; the norm's gradient is linear in dY, its arithmetic within
2^-18 of the magnitudes, and its result is rounded.  The sums of absolute values make the bound wide, so the test also asks that each
branch of the gradient is larger than the bound, i.e. that losing one would be seen."""
import pytest
import torch

from tests.test_gpu_block_norm import ARITH, EPS, _std
from tests.test_gpu_ffn_block import decoded, example  # noqa: F401
from tests.test_gpu_linear_act import FN, TOL, act64

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.mark.parametrize("tokens,hidden,inner", [(3, 256, 512), (40, 512, 1088), (200, 768, 1024)])
def test_gradient_of_the_block_against_the_formula(example, tokens, hidden, inner):      # noqa: F811
    import paper_2602_11287_b200 as hif4
    block = example.FeedForward(hidden, inner, seed=3)
    g = torch.Generator(device="cuda"); g.manual_seed(tokens)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    x, r, dout = rnd(tokens, hidden), rnd(tokens, hidden), rnd(tokens, hidden)
    w = (1 + 0.1 * rnd(hidden).float()).to(torch.bfloat16)
    leaves = [t.clone().requires_grad_() for t in (x, r, w)]
    block(*leaves).backward(dout)
    h, y, _ = block.forward(x, r, w)
    Y, G, Up, D = (decoded(hif4, t) for t in (y, block.gate, block.up, block.down))
    H, W, DO = h.double().requires_grad_(), w.double().requires_grad_(), dout.double()

    df = DO @ D
    e_df = U * df.abs() + TOL * (DO.abs() @ D.abs())
    gate, up = Y @ G.t(), Y @ Up.t()
    e_gate, e_up = TOL * (Y.abs() @ G.abs().t()), TOL * (Y.abs() @ Up.abs().t())
    a, s = act64(gate, 2)
    e_a, e_s = 1.2 * e_gate + FN * a.abs(), 2 * e_gate + FN * (s.abs() + gate.abs())
    dg, du = df * up * s, df * a
    far_up, far_s, far_a = up.abs() + e_up, s.abs() + e_s, a.abs() + e_a
    e_dg = e_df * far_up * far_s + df.abs() * (e_s * far_up + s.abs() * e_up)
    e_du = e_df * far_a + df.abs() * e_a
    e_dg, e_du = ((1 + U) * e + U * v.abs() for e, v in ((e_dg, dg), (e_du, du)))
    dy = dg @ G + du @ Up
    e_dy = e_dg @ G.abs() + e_du @ Up.abs() + TOL * (dg.abs() @ G.abs() + du.abs() @ Up.abs())
    e_dy = (1 + U) * e_dy + U * dy.abs()

    dh, dw = torch.autograd.grad(_std(H, 1) * W, [H, W], dy)
    want = DO + dh
    H, W = H.detach(), W.detach()
    n, rstd = _std(H, 1).abs(), 1.0 / torch.sqrt((H * H).mean(1, keepdim=True) + EPS)
    through = lambda e: rstd * (e * W.abs() + n * (e * W.abs() * n).mean(1, keepdim=True))        # noqa: E731
    mag = DO.abs() + rstd * (dy.abs() * W.abs()).amax(1, keepdim=True) * (1 + n * n.amax(1, keepdim=True))
    bound = U * want.abs() + through(e_dy) + ARITH * mag
    bound_w = (e_dy * n).sum(0) + 2.0 ** -24 * (64 + tokens / 148 + 300) * (dy.abs() * n).sum(0) + U * dw.abs()        # (rounded to BF16 by the caller)
    gx, gr, gw = (t.grad.double() for t in leaves)
    for got, ref, b in ((gx, want, bound), (gr, want, bound), (gw, dw, bound_w)):
        assert bool(((got - ref).abs() <= b).all()), float(((got - ref).abs() / b).max())

    for branch in (dg @ G, du @ Up):
        assert float(through(branch).norm()) > float(bound.norm()) and float(torch.autograd.grad(
            (_std(H.requires_grad_(), 1) * W), [H], branch)[0].norm()) > float(bound.norm())
        if tokens < 10:                  # (over many tokens the branch's signs average out, the bound's sums do not)
            assert float((branch * _std(H.detach(), 1)).sum(0).norm()) > float(bound_w.norm())
