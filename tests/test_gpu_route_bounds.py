"""Routing where FP32 cannot tell groups apart: sums of two choices that cancel or overflow, scores next to the error bound."""
import math

import pytest
import torch

from tests.test_gpu_experts import SIGMOID, SOFTMAX, check_route, gen, hif4  # noqa: F401  (hif4: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bias,logits,kept", [
    ([65536.0, -65536.0, 65536.0, -65536.0], [1.441, -1.237, -0.774, 0.967], 1),
    ([1000.0, -1000.0, 1000.0, -1000.0], [-6.648e-5, -5.265e-5, -1.2645e-4, 5.188e-5], 1)])
def test_a_cancelling_sum_of_two(hif4, bias, logits, kept):  # noqa: F811
    """The sums of the groups differ by less than FP32 keeps of their terms: the second group's is larger in 64 bits."""
    x, b = torch.tensor([logits], device="cuda"), torch.tensor(bias, device="cuda")
    ids, _ = check_route(hif4, x, 2, b, score=SIGMOID, groups=2, top_groups=kept, group_best=2)
    assert ids.tolist() == [[2, 3]]


# (E, groups): groups of whole lanes, of several lanes, of parts of lanes, many experts a lane
@pytest.mark.parametrize("E,groups,kept,k", [(4, 2, 1, 2), (256, 8, 4, 8), (512, 8, 4, 6), (160, 8, 3, 6), (96, 32, 5, 4), (775, 31, 9, 12), (1024, 4, 2, 32)])
@pytest.mark.parametrize("size", [1.0, 16.0, 256.0, 4096.0, 65536.0])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_groups_with_biases_of_both_signs(hif4, E, groups, kept, k, size, score):  # noqa: F811
    """One expert of a group with a bias of +size, the others with -size."""
    g = gen(E + int(size))
    per = E // groups
    bias = torch.full((groups, per), -size, device="cuda")
    bias.scatter_(1, torch.randint(0, per, (groups, 1), generator=g, device="cuda"), size)
    for spread in (1.0, size * 2.0 ** -18):                # and logits whose scores differ by about the rounding of such a bias
        logits = spread * torch.randn(4000, E, generator=g, device="cuda")
        for best in (1, 2):
            check_route(hif4, logits, k, bias.view(-1), score=score, groups=groups, top_groups=kept, group_best=best)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_a_kept_group_of_large_terms(hif4, score):  # noqa: F811
    """Not the last kept group but the first one has the terms that FP32 cannot hold."""
    g = gen(7)
    E, groups, per = 64, 8, 8
    bias = torch.zeros(groups, per, device="cuda")
    bias[2, 1], bias[2, 2:] = 2.0 ** 17, -(2.0 ** 17)
    bias[2, 0] = -(2.0 ** 17)
    logits = 2.0 ** -6 * torch.randn(4000, E, generator=g, device="cuda")
    check_route(hif4, logits, 8, bias.view(-1), score=score, groups=groups, top_groups=3, group_best=2)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("E,groups", [(6, 3), (256, 8), (160, 8), (96, 32)])
def test_groups_masked_by_the_lowest_value(hif4, score, E, groups):  # noqa: F811
    """Experts masked by FP32's lowest value can be chosen, those masked by -inf cannot: a group's sum of two lowest values is no -inf.
    Sums of two largest values are no +inf either."""
    g = gen(E)
    per = E // groups
    low = torch.finfo(torch.float32).min
    logits = torch.randn(50, E, generator=g, device="cuda")
    for fills in ((-math.inf, low, 0.0), (low, -math.inf, 0.0), (low, low, -math.inf), (-low, -low, 0.0), (0.0, -low, -low)):
        bias = torch.zeros(groups, per, device="cuda")
        for at, fill in enumerate(fills):
            bias[at] = fill
        bias[3:] = -math.inf
        for kept in (1, 2, 3):
            ids, _ = check_route(hif4, logits, min(2 * kept, 8), bias.view(-1), score=score, groups=groups, top_groups=kept, group_best=2)
    bias = torch.full((groups, per), -math.inf, device="cuda")
    bias[1], bias[2] = low, 0.0
    ids, _ = check_route(hif4, logits, 4, bias.view(-1), score=score, groups=groups, top_groups=2, group_best=2)
    if per == 2:                                           # the third group's two, then the second's
        assert bool((ids[:, :2] >= 4).all()) and bool(((ids[:, 2:] == 2) | (ids[:, 2:] == 3)).all())


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_groups_with_infinite_biases(hif4, score):  # noqa: F811
    """An expert with a bias of +inf is chosen first, and so is its group; several such go by index."""
    g = gen(11)
    logits = torch.randn(300, 256, generator=g, device="cuda")
    bias = 0.1 * torch.randn(256, generator=g, device="cuda")
    for places in ([5], [5, 6], [5, 100], [5, 100, 200, 250]):
        b = bias.clone()
        b[places] = math.inf
        for best in (1, 2):
            for kept in (1, 3):
                check_route(hif4, logits, 8, b, score=score, groups=8, top_groups=kept, group_best=best)


@pytest.mark.parametrize("E,k", [(256, 8), (512, 8), (1024, 32)])
def test_softmax_choices_next_to_the_error_bound(hif4, E, k):  # noqa: F811
    """Biases that bring experts of different scores within a few 2^-22 of the largest score of one another, among many terms whose
    rounded sum is off."""
    g = gen(E)
    depth = -7.0 - torch.rand(3000, 1, generator=g, device="cuda")
    logits = depth.expand(-1, E).clone()
    logits[:, 0] = 0.0
    total = 1.0 + (E - 1) * depth[0, 0].double().exp()
    bias = torch.zeros(E, device="cuda")
    for n in range(1, k):                                  # expert n against the first: its bias makes up for the difference, nearly
        bias[n] = ((1.0 - depth[0, 0].double().exp()) / total * (1.0 + (n - k // 2) * 2.0 ** -22)).float()
    check_route(hif4, torch.cat([logits[:1].expand(3000, -1) + 2.0 ** -24 * torch.randn(3000, E, generator=g, device="cuda"), logits]), k, bias, score=SOFTMAX)
