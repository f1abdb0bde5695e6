"""Routing's neighbours and 4-bit products past 2^31 elements: the ends of the matrices are where 32-bit offsets would go wrong."""
import pytest
import torch

from tests import bfp4_reference as ref
from tests.test_gpu_bfp4 import check_product

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hif4():
    import paper_2602_11287_b200 as m
    return m


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


ENDS = [slice(0, 3), slice(-3, None)]


@pytest.mark.parametrize("fmt", [1, 2])
def test_conversion(hif4, fmt):
    rows, cols = 524291, 4160
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:], x[-3:] = 1.0, torch.randn(3, cols, device="cuda")
    x[:3] = torch.randn(3, cols, device="cuda")
    codes, scales = hif4.hif4_bfp4_quantize(x, fmt)
    back = hif4.hif4_bfp4_dequantize((codes, scales), fmt)
    for e in ENDS:
        want = hif4.hif4_bfp4_quantize(x[e], fmt)
        assert torch.equal(codes[e], want[0]) and torch.equal(scales[:, e], want[1])
        assert torch.equal(back[e], hif4.hif4_bfp4_dequantize(want, fmt))


def test_conversion_down_the_columns(hif4):
    rows, cols = 4160, 524296
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:, -8:], x[:, :8] = torch.randn(rows, 8, device="cuda"), torch.randn(rows, 8, device="cuda")
    codes, scales = hif4.hif4_bfp4_quantize_transposed(x, 2)
    for e in (slice(0, 8), slice(-8, None)):
        want = hif4.hif4_bfp4_quantize(x[:, e].t().contiguous(), 2)
        assert torch.equal(codes[e], want[0]) and torch.equal(scales[:, e], want[1])


@pytest.mark.parametrize("grouped", [False, True])
def test_product(hif4, grouped):
    M, N, K = 262150, 8256, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    a, b = ref.random_operand(M, K, 2, g), ref.random_operand(N, K, 2, g, groups=2 if grouped else None)
    B = ref.values(*b, 2)
    if grouped:
        y = hif4.hif4_bfp4_grouped_gemm(a, b, torch.tensor([0, 5, M], device="cuda"), 2)
    else:
        y = hif4.hif4_bfp4_gemm(a, b, 2)
    for e, which in ((slice(0, 3), 0), (slice(M - 3, M), 1)):
        check_product(y[e], ref.values(a[0][e], a[1][:, e], 2), B[which] if grouped else B)


def test_rows_of_experts_and_their_sum(hif4):
    T, k, K = 40000, 8, 7168
    x = torch.ones(T, K, dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn(2, K, device="cuda")
    ids = torch.full((T, k), 3, dtype=torch.int32, device="cuda")        # one expert many times: the last token's rows are the last
    off, row_of = hif4.hif4_expert_plan(ids, 4)
    assert off.tolist() == [0, 0, 0, 0, T * k] and row_of[-1].tolist() == list(range(T * k - k, T * k))
    rows = hif4.hif4_dispatch(x, row_of)
    assert torch.equal(rows[-k:], x[-1:].expand(k, K)) and torch.equal(rows[:k], x[:1].expand(k, K))
    units = hif4.hif4_dispatch(x, row_of, fmt=0)
    assert torch.equal(units[-k:], hif4.hif4_quantize(x[-1:]).expand(k, -1, -1))
    w = torch.full((T, k), 0.125, device="cuda")
    assert torch.equal(hif4.hif4_combine(rows, row_of, w)[-2:], x[-2:])
    d, dw = hif4.hif4_combine_backward(x, row_of, w, rows=rows)
    assert torch.equal(d[-k:].float(), (0.125 * x[-1:].float()).expand(k, K))
    want = (x[-1].double() ** 2).sum()
    assert bool(((dw[-1].double() - want).abs() <= 1e-5 * want).all())


def test_routing_of_many_tokens(hif4):
    T, E = 4200000, 512
    logits = torch.zeros(T, E, dtype=torch.bfloat16, device="cuda")
    logits[-1, 300], logits[-1, 7], logits[0, 9] = 4.0, 3.0, 5.0
    ids, w = hif4.hif4_route(logits, 2)
    assert ids[-1].tolist() == [300, 7] and ids[0].tolist() == [9, 0] and ids[1].tolist() == [0, 1]
    d = hif4.hif4_route_backward(torch.tensor([[1.0, 0.0]], device="cuda").expand(T, 2).contiguous(), logits, ids)
    p = float(w[-1, 0])
    assert abs(float(d[-1, 300]) - p * (1 - p)) < 2.0 ** -9 and float(d[-1].float().abs().sum()) > 0 and bool((d[-1, 301:] == 0).all())
