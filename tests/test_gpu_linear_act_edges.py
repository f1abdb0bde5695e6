"""hif4_linear_act, hif4_gated_linear and their gradients at the edges of their arguments: a single row with any stride,
infinite and NaN gradients, more rows than a grid has blocks, activations without the slack of a product, captured graphs.

Tolerances as in test_gpu_linear_act.py; an activation alone is within (8 + 2 |e|) 2^-22 of its value, e the exponent that its
formula has (-z, z^2 / 2, or twice the argument of tanh): two units of 2^-23 for each of the exponential, the division and the
roundings around them, and e times the rounding of the exponent itself.  A sigmoid below 2^-126 is zero."""
import pytest
import torch

from tests.test_gpu_linear_act import FN, TINY, TOL, TYPES, U, act64, call, close, decode, expect_forward, hif4, operands  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------- a single row
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [320, 1024])
@pytest.mark.parametrize("pad", [1, 4, 13])
def test_one_row_of_any_stride(hif4, gated, dtype, K, pad):
    """A single row has no next one: its stride does not matter, whatever kernel takes it."""
    x, w, b = operands(hif4, 1, 192, K, dtype, gated, K + pad)
    wide = torch.zeros(3, K + pad, dtype=dtype, device="cuda")
    row = wide[:1, :K]
    row.copy_(x)
    assert row.stride(0) == K + pad
    assert torch.equal(call(hif4, row, w, b, act=2), call(hif4, x, w, b, act=2))
    assert torch.equal(call(hif4, row, w, b, act=2, units=True, dtype=dtype), call(hif4, x, w, b, act=2, units=True, dtype=dtype))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", [320, 1024])
def test_gradient_of_one_row_of_any_stride(hif4, gated, dtype, K):
    x, w, b = operands(hif4, 1, 192, K, dtype, gated, K)
    wide = torch.zeros(3, K + 5, dtype=dtype, device="cuda")
    row = wide[:1, :K]
    row.copy_(x)
    dy = torch.randn(1, 192, device="cuda").to(dtype)
    f = hif4.hif4_gated_linear_backward if gated else hif4.hif4_linear_act_backward
    got, want = (f(dy, t, *w, *b, act=2, want_dbias=True) for t in (row, x))
    assert all(torch.equal(g, v) for g, v in zip(got, want))
