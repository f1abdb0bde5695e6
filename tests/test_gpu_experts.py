"""Routing to experts, the experts' rows and their combination against the definitions in 64 bits."""
import math

import pytest
import torch

from tests import bfp4_reference as ref

pytestmark = pytest.mark.gpu
SOFTMAX, SIGMOID = 0, 1


@pytest.fixture(scope="module")
def hif4():
    import paper_2602_11287_b200 as m
    return m


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def choices(logits, bias, score, sums):
    x = logits.double()
    if bias is None and not sums:
        c = x
    else:
        high = x.nan_to_num(nan=-math.inf).amax(1, keepdim=True)
        p = torch.where(x == high, 1.0, torch.exp(x - high)).nan_to_num(nan=0.0) * (high > -math.inf)
        c = torch.sigmoid(x) if score == SIGMOID else p / p.sum(1, keepdim=True).clamp(min=1e-300)
        if bias is not None:
            c = c + bias.double()
        c = torch.where(x == -math.inf, -math.inf, c)
    return torch.where(x.isnan() | c.isnan(), -math.inf, c)


def route(logits, k, bias=None, score=SOFTMAX, groups=1, top_groups=None, group_best=1, renormalize=True, scale=1.0):
    T, E = logits.shape
    c = choices(logits, bias, score, groups > 1 and group_best == 2)
    if groups > 1:
        per = c.view(T, groups, -1)
        value = per.sort(dim=2, descending=True)[0][..., :group_best].sum(2)
        best = value.sort(dim=1, descending=True, stable=True)[1][:, : top_groups or groups]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, best, True)
        c = torch.where(keep.unsqueeze(2), per, -math.inf).view(T, E)
    order = c.sort(dim=1, descending=True, stable=True)
    ids = torch.where(order[0][:, :k] > -math.inf, order[1][:, :k], -1)
    x = logits.double()
    s = torch.sigmoid(x) if score == SIGMOID else torch.softmax(x, 1)
    w = torch.where(ids >= 0, s.gather(1, ids.clamp(min=0)), 0.0)
    if renormalize:                                        # by logarithms: every score of a row may be below what 64 bits hold
        l = torch.where(ids >= 0, (torch.nn.functional.logsigmoid(x) if score == SIGMOID else x).gather(1, ids.long().clamp(min=0)), -math.inf)
        w = torch.where(ids >= 0, torch.softmax(l, 1), 0.0)
    bad = x.isnan().any(1) | (x == math.inf).any(1) if score == SOFTMAX else x.isnan().any(1)
    return ids.int(), torch.where(bad.unsqueeze(1), math.nan, scale * w)


def check_route(hif4, logits, k, bias=None, **kw):
    ids, w = hif4.hif4_route(logits, k, bias, **kw)
    want = route(logits, k, bias, **kw)
    assert torch.equal(ids, want[0])
    # FP32: the exponential's argument is off by 2^-24 of up to 100, exponential, sums of up to 1024 terms in a tree, two divisions
    assert torch.equal(w.isnan(), want[1].isnan())
    assert bool(((w.double() - want[1]).nan_to_num(0.0).abs() <= 2.0 ** -18 * want[1].nan_to_num(0.0).abs() + 1e-37).all())
    return ids, w


SHAPES = [(1, 1, 1), (1, 256, 8), (5, 7, 7), (33, 33, 2), (100, 64, 6), (129, 100, 16), (64, 512, 10), (17, 1000, 32), (9, 1024, 1)]


@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_route(hif4, T, E, k, score, dtype):
    g = gen(T + E + k)
    logits = (2.0 * torch.randn(T, E, generator=g, device="cuda")).to(dtype)
    bias = 0.1 * torch.randn(E, generator=g, device="cuda")
    for b in (None, bias):
        for renorm in (False, True):
            check_route(hif4, logits, k, b, score=score, renormalize=renorm, scale=2.5)


@pytest.mark.parametrize("E,groups,kept,k", [(256, 8, 4, 8), (64, 8, 3, 6), (64, 32, 5, 5), (96, 3, 2, 10), (1024, 4, 1, 20), (160, 8, 8, 6), (12, 6, 2, 4)])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_with_groups(hif4, E, groups, kept, k, best, score):
    g = gen(E + groups)
    for dtype in (torch.float32, torch.bfloat16):
        logits = torch.randn(70, E, generator=g, device="cuda").to(dtype)
        bias = 0.1 * torch.randn(E, generator=g, device="cuda")
        for b in (None, bias):
            check_route(hif4, logits, k, b, score=score, groups=groups, top_groups=kept, group_best=best)


def test_route_equal_scores_and_close_ones(hif4):
    """Equal ones go by index; neighbours closer than FP32 tells apart keep the order of their values."""
    logits = torch.zeros(4, 256, device="cuda")
    logits[1, 100:] = 1.0
    logits[2] = torch.arange(256, device="cuda") % 3
    logits[3] = 30.0                                       # one in FP32 as a sigmoid
    logits[3, 77], logits[3, 200] = 31.0, 30.5
    bias = torch.zeros(256, device="cuda")
    for kw in (dict(), dict(groups=8, top_groups=3, group_best=2)):
        for b in (None, bias):
            for score in (SOFTMAX, SIGMOID):
                check_route(hif4, logits, 8, b, score=score, **kw)
    ids, _ = hif4.hif4_route(logits, 3, bias, score=SIGMOID)
    assert ids.tolist() == [[0, 1, 2], [100, 101, 102], [2, 5, 8], [77, 200, 0]]
    g = gen(3)
    base = torch.randn(300, 1, generator=g, device="cuda")
    close = base + torch.randint(0, 8, (300, 64), generator=g, device="cuda") * 2.0 ** -23
    check_route(hif4, close, 8, 0.5 + torch.zeros(64, device="cuda"), score=SIGMOID)
    check_route(hif4, close, 8, torch.randn(64, generator=g, device="cuda") * 2.0 ** -24, score=SIGMOID, groups=4, top_groups=2, group_best=2)
    check_route(hif4, close, 8, torch.randn(64, generator=g, device="cuda") * 2.0 ** -30, score=SOFTMAX)


@pytest.mark.parametrize("E,groups,kept,k", [(256, 1, 1, 8), (256, 8, 4, 8), (40, 1, 1, 32), (32, 1, 1, 32), (168, 8, 7, 15), (66, 2, 1, 9), (775, 31, 5, 32), (96, 32, 3, 6)])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_few_values(hif4, E, groups, kept, k, score):
    """Logits and biases of few values: most neighbours are equal, and some equal sums are of different terms."""
    g = gen(E + k)
    logits = torch.randint(-6, 7, (200, E), generator=g, device="cuda").bfloat16() / 4
    bias = torch.randint(0, 3, (E,), generator=g, device="cuda") / 64.0
    for b in (None, bias, torch.zeros_like(bias)):
        for best in (1, 2):
            check_route(hif4, logits, k, b, score=score, groups=groups, top_groups=kept, group_best=best)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_masked_and_special_logits(hif4, score):
    g = gen(9)
    logits = torch.randn(12, 64, generator=g, device="cuda")
    logits[0] = -math.inf
    logits[1, 3:] = -math.inf
    logits[2, 5] = math.nan
    logits[3, 6] = math.inf
    logits[4] = torch.finfo(torch.float32).min
    logits[5, ::2] = torch.finfo(torch.float32).min
    logits[6] = math.nan
    logits[7] *= 1e30
    logits[8] -= 200.0                                     # sigmoids far below FP32
    bias = 0.1 * torch.randn(64, generator=g, device="cuda")
    masked = bias.clone()
    masked[10:60] = -math.inf
    for b in (None, bias, masked):
        for kw in (dict(), dict(groups=8, top_groups=2, group_best=2), dict(groups=4, top_groups=4)):
            ids, w = check_route(hif4, logits[[0, 1, 2, 3, 4, 5, 6, 9, 10, 11]], 8, b, score=score, **kw)
            assert ids[0].tolist() == [-1] * 8 and w[0].tolist() == [0.0] * 8
    ids, w = hif4.hif4_route(logits[8:9], 8, score=score)
    assert bool((w.double() - torch.softmax(logits[8].double()[ids[0].long()], 0)).abs().max() < 1e-5)   # e^x / (1 + e^x) = e^x here


@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_route_gradient(hif4, T, E, k, score, dtype):
    g = gen(T * E)
    logits = torch.randn(T, E, generator=g, device="cuda").to(dtype)
    dw = torch.randn(T, k, generator=g, device="cuda")
    for renorm in (False, True):
        ids, _ = hif4.hif4_route(logits, k, score=score, renormalize=renorm, scale=1.5)
        ids[0, k // 2] = -1
        if T > 2:
            ids[2] = -1
        got = hif4.hif4_route_backward(dw, logits, ids, score=score, renormalize=renorm, scale=1.5)
        x = logits.double().requires_grad_()
        s = torch.sigmoid(x) if score == SIGMOID else torch.softmax(x, 1)
        w = torch.where(ids >= 0, s.gather(1, ids.long().clamp(min=0)), 0.0)
        if renorm:
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        want, = torch.autograd.grad(1.5 * w, x, dw.double())
        size = (1.5 * dw.abs()).amax(1, keepdim=True).double()
        assert got.dtype == dtype
        half = torch.finfo(dtype).eps / 2
        # FP32 terms of size |dw| cancel: 2^-18 of the largest, and one rounding
        assert bool(((got.double() - want).abs() <= half * want.abs() + 2.0 ** -18 * size).all())


def test_route_gradient_against_differences(hif4):
    g = gen(4)
    logits = torch.randn(6, 30, generator=g, device="cuda")
    dw = torch.randn(6, 5, generator=g, device="cuda")
    for score in (SOFTMAX, SIGMOID):
        for renorm in (False, True):
            ids, _ = hif4.hif4_route(logits, 5, score=score, renormalize=renorm)
            d = hif4.hif4_route_backward(dw, logits, ids, score=score, renormalize=renorm)
            step = torch.randn(6, 30, generator=g, device="cuda") * 2.0 ** -7
            f = []
            for sign in (1, -1):
                i2, w2 = hif4.hif4_route(logits + sign * step, 30, score=score, renormalize=False)
                at = torch.zeros_like(w2).scatter_(1, i2.long(), w2).gather(1, ids.long())
                f.append((dw * (at / at.sum(1, keepdim=True) if renorm else at)).sum(1))
            slope, want = (d * step).sum(1), (f[0] - f[1]) / 2
            # differences: third order (2^-7)^3 x the size of what is summed, and FP32 in f
            assert bool(((slope - want).abs() <= 1e-4 * dw.abs().sum(1)).all())


def test_route_of_a_view_and_no_tokens(hif4):
    wide = torch.randn(20, 90, device="cuda")
    a, b = hif4.hif4_route(wide[:, 10:74], 4), hif4.hif4_route(wide[:, 10:74].contiguous(), 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ids, w = hif4.hif4_route(wide[:0], 4)
    assert ids.shape == (0, 4) and w.shape == (0, 4)
    assert hif4.hif4_route_backward(w, wide[:0], ids).shape == (0, 90)


def plan(ids, E):
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    order = key.argsort(stable=True)
    row = torch.empty_like(order)
    row[order] = torch.arange(flat.numel(), device=ids.device)
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=ids.device), torch.bincount(key, minlength=E + 1)[:E].cumsum(0)])
    return off, torch.where(key < E, row, -1).view(ids.shape).int()


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 256), (3, 5, 7), (1000, 8, 256), (1024, 8, 1024), (1025, 8, 64), (5000, 6, 100), (70000, 2, 33), (512, 8, 1024), (513, 8, 300), (300000, 8, 64),
                                   (4096, 8, 1)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_plan(hif4, T, k, E, drop):
    g = gen(T + E)
    ids = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)            # the same expert twice, too
    if drop:
        ids[torch.rand(T, k, generator=g, device="cuda") < drop] = -1
        ids[T // 2, 0] = E
        ids[T // 3, -1] = 2 ** 31 - 1
        ids[0, 0] = -(2 ** 31)
    off, row_of = hif4.hif4_expert_plan(ids, E)
    want = plan(ids, E)
    assert torch.equal(off, want[0]) and torch.equal(row_of, want[1])


def test_plan_of_no_tokens_and_of_padding_only(hif4):
    off, row_of = hif4.hif4_expert_plan(torch.empty(0, 4, dtype=torch.int32, device="cuda"), 9)
    assert off.tolist() == [0] * 10 and row_of.shape == (0, 4)
    off, row_of = hif4.hif4_expert_plan(torch.full((30, 2), -1, dtype=torch.int32, device="cuda"), 9)
    assert off.tolist() == [0] * 10 and bool((row_of == -1).all())


def assignment(T, k, E, seed, drop=0.1):
    g = gen(seed)
    ids = torch.rand(T, E, generator=g, device="cuda").argsort(1)[:, :k].int().contiguous()
    ids[torch.rand(T, k, generator=g, device="cuda") < drop] = -1
    return ids


@pytest.mark.parametrize("T,k,K", [(1, 1, 64), (1, 8, 7168), (5, 3, 192), (130, 6, 1088), (600, 2, 64), (1500, 2, 9280)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_dispatch(hif4, T, k, K, dtype):
    x = (torch.randn(T, K, generator=gen(T + K), device="cuda") * 3).to(dtype)
    off, row_of = hif4.hif4_expert_plan(assignment(T, k, 16, T), 16)
    at = row_of[row_of >= 0].long()
    token = torch.arange(T, device="cuda").unsqueeze(1).expand(T, k)[row_of >= 0]
    R = T * k
    out = torch.full((R, K), 5.0, dtype=dtype, device="cuda")
    want = out.clone()
    want[at] = x[token]
    assert hif4.hif4_dispatch(x, row_of, out=out) is out and torch.equal(out, want)
    for mode in (hif4.HIF4_RNE, hif4.HIF4_RHA):
        units = torch.full((R, K // 64, 36), 7, dtype=torch.uint8, device="cuda")
        want = units.clone()
        want[at] = hif4.hif4_quantize(x, mode)[token]
        assert torch.equal(hif4.hif4_dispatch(x, row_of, fmt=hif4.HIF4_FMT_HIF4, mode=mode, out=units), want)
    for fmt in (hif4.HIF4_FMT_MXFP4, hif4.HIF4_FMT_NVFP4):
        for gain in (None, torch.full((1,), 0.7, device="cuda")):
            q = hif4.hif4_bfp4_quantize(x, fmt, gain=gain)
            out = torch.full((R, K // 2), 7, dtype=torch.uint8, device="cuda"), torch.full((q[1].shape[0], R, 16), 7, dtype=torch.uint8, device="cuda")
            codes, scales = out[0].clone(), out[1].clone()
            codes[at], scales[:, at] = q[0][token], q[1][:, token]
            got = hif4.hif4_dispatch(x, row_of, fmt=fmt, gain=gain, out=out)
            assert torch.equal(got[0], codes) and torch.equal(got[1], scales)


@pytest.mark.parametrize("K,shift", [(1, 0), (7, 0), (66, 1), (1000, 3), (2056, 0)])
def test_dispatch_rows_of_any_length_and_address(hif4, K, shift):
    wide = torch.randn(40, K + 9, generator=gen(K), device="cuda").to(torch.bfloat16)
    x = wide[:, shift:shift + K]
    off, row_of = hif4.hif4_expert_plan(assignment(40, 3, 8, 1), 8)
    got = hif4.hif4_dispatch(x, row_of)
    at = row_of[row_of >= 0].long()
    token = torch.arange(40, device="cuda").unsqueeze(1).expand(40, 3)[row_of >= 0]
    assert torch.equal(got[at], x[token])


def test_rows_outside_the_output_are_left_out(hif4):
    """Row numbers that the output does not have reach no memory."""
    x = torch.randn(6, 128, device="cuda").to(torch.bfloat16)
    row_of = torch.tensor([[0, -1], [1, 9], [2, 2 ** 31 - 1], [3, -(2 ** 31)], [4, 5], [6, 7]], dtype=torch.int32, device="cuda")
    pool = torch.full((20, 128), 4.0, dtype=torch.bfloat16, device="cuda")
    hif4.hif4_dispatch(x, row_of, out=pool[:5])
    assert torch.equal(pool[:5], x[:5]) and bool((pool[5:] == 4.0).all())
    y = hif4.hif4_combine(pool[:5], row_of)
    assert torch.equal(y[:5], x[:5]) and bool((y[5] == 0).all())
    d, dw = hif4.hif4_combine_backward(x, row_of, rows=pool[:5])
    assert torch.equal(d, x[:5]) and bool((dw[1:, 1] == 0).all() and (dw[5] == 0).all())


TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("T,k,K,pad", [(1, 8, 7168, 0), (1, 1, 1, 0), (40, 6, 2056, 0), (33, 9, 1001, 0), (200, 4, 64, 8), (50, 32, 320, 3), (700, 3, 2056, 0), (300, 5, 777, 0), (90, 4, 1002, 2)])
@pytest.mark.parametrize("dt_in", TYPES)
@pytest.mark.parametrize("dt", TYPES)
def test_combine_and_its_gradient(hif4, T, k, K, pad, dt_in, dt):
    g = gen(T + K + k)
    off, row_of = hif4.hif4_expert_plan(assignment(T, k, 40, T + 1), 40)
    R = T * k
    rows = torch.randn(R, K + pad, generator=g, device="cuda").to(dt_in)[:, :K]
    w = torch.randn(T, k, generator=g, device="cuda")
    res = torch.randn(T, K + pad, generator=g, device="cuda").to(dt)[:, :K]
    dy = torch.randn(T, K + pad, generator=g, device="cuda").to(dt)[:, :K]
    there = (row_of >= 0).unsqueeze(-1)
    picked = torch.where(there, rows[row_of.long().clamp(min=0)].double(), 0.0)
    half = torch.finfo(dt).eps / 2
    for weights, r in ((w, res), (None, None), (w, None)):
        W = torch.ones_like(w) if weights is None else w
        terms = picked * W.double().unsqueeze(-1)
        want, size = terms.sum(1), terms.abs().sum(1)
        if r is not None:
            want, size = want + 0.5 * r.double(), size + 0.5 * r.double().abs()
        y = hif4.hif4_combine(rows, row_of, weights, residual=r, res_scale=0.5, dtype=dt)
        # k + 1 fused multiply-adds, then one rounding
        assert y.dtype == dt and bool(((y.double() - want).abs() <= (k + 1) * 2.0 ** -24 * size + half * want.abs() + 2.0 ** -25).all())
        out = torch.full((R, K), 8.0, dtype=dt_in, device="cuda")
        d, dw = hif4.hif4_combine_backward(dy, row_of, weights, rows=rows, out=out)
        each = dy.double().unsqueeze(1) * W.double().unsqueeze(-1)
        want_d = torch.full((R, K), 8.0, dtype=torch.float64, device="cuda")
        want_d[row_of[row_of >= 0].long()] = each[row_of >= 0]
        assert d is out and bool(((d.double() - want_d).abs() <= (2.0 ** -24 + torch.finfo(dt_in).eps / 2) * want_d.abs() + 2.0 ** -25).all())
        prod = picked * dy.double().unsqueeze(1)
        assert bool(((dw.double() - prod.sum(-1)).abs() <= (K + 16) * 2.0 ** -24 * prod.abs().sum(-1) + 1e-37).all())
    only, none = hif4.hif4_combine_backward(dy, row_of, w, num_rows=R, dtype=dt_in)
    assert none is None and torch.equal(only[row_of[row_of >= 0].long()], hif4.hif4_combine_backward(dy, row_of, w, rows=rows)[0][row_of[row_of >= 0].long()])
    assert hif4.hif4_combine_backward(dy, row_of, w, rows=rows, want_drows=False)[0] is None


def test_combine_over_its_residual(hif4):
    off, row_of = hif4.hif4_expert_plan(assignment(60, 4, 8, 2), 8)
    rows, r = torch.randn(240, 512, device="cuda"), torch.randn(60, 512, device="cuda").to(torch.bfloat16)
    want = hif4.hif4_combine(rows, row_of, residual=r)
    assert hif4.hif4_combine(rows, row_of, residual=r, out=r) is r and torch.equal(r, want)


def test_gradient_of_dispatch_is_combine(hif4):
    """<dispatch(x), d> = <x, combine(d)> for whole numbers, where sums are exact."""
    g = gen(5)
    off, row_of = hif4.hif4_expert_plan(assignment(50, 5, 8, 3), 8)
    x = torch.randint(-8, 9, (50, 96), generator=g, device="cuda").float()
    d = torch.randint(-8, 9, (250, 96), generator=g, device="cuda").float()
    out = hif4.hif4_dispatch(x, row_of, out=torch.zeros(250, 96, device="cuda"))
    assert float((out * d).sum()) == float((x * hif4.hif4_combine(d, row_of)).sum())


def test_refusals(hif4):
    x, ids = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    w = torch.zeros(4, 2, device="cuda")
    big = torch.zeros(2, 1025, device="cuda")
    before = hif4.launch_count()
    for f, code in ((lambda: hif4.hif4_route(x, 0), 2), (lambda: hif4.hif4_route(x, 65), 2), (lambda: hif4.hif4_route(x, 33), 8),
                    (lambda: hif4.hif4_route(big, 2), 8), (lambda: hif4.hif4_route(x, 2, score=2), 4), (lambda: hif4.hif4_route(x, 2, score=2 ** 32), 4),
                    (lambda: hif4.hif4_route(x, 2, groups=3), 2), (lambda: hif4.hif4_route(x, 2, groups=0), 2),
                    (lambda: hif4.hif4_route(x, 2, groups=8, top_groups=9), 2), (lambda: hif4.hif4_route(x, 9, groups=8, top_groups=1), 2),
                    (lambda: hif4.hif4_route(x, 2, groups=64), 8), (lambda: hif4.hif4_route(x, 2, groups=8, group_best=3), 2),
                    (lambda: hif4.hif4_route(x, 2, groups=0), 2), (lambda: hif4.hif4_route_backward(w, x, ids, score=-1), 4),
                    (lambda: hif4.hif4_expert_plan(ids, 0), 2), (lambda: hif4.hif4_expert_plan(ids, 1025), 8),
                    (lambda: hif4.hif4_dispatch(x, ids, fmt=3), 4), (lambda: hif4.hif4_dispatch(x, ids, fmt=0, mode=2), 4),
                    (lambda: hif4.hif4_dispatch(x[:, :60], ids, fmt=0), 2),
                    (lambda: hif4.hif4_dispatch(torch.zeros(4, 65, device="cuda")[:, 1:], ids, fmt=0), 3)):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        assert e.value.code == code
    for f in (lambda: hif4.hif4_route(x.cpu(), 2), lambda: hif4.hif4_route(x, 2, torch.zeros(63, device="cuda")), lambda: hif4.hif4_route(x.t(), 2),
              lambda: hif4.hif4_route(x, 2, torch.zeros(64, device="cuda", dtype=torch.bfloat16)), lambda: hif4.hif4_expert_plan(ids.long(), 4),
              lambda: hif4.hif4_expert_plan(ids.t(), 4), lambda: hif4.hif4_dispatch(x, ids[:3]), lambda: hif4.hif4_dispatch(x, ids, out=x.double()),
              lambda: hif4.hif4_dispatch(x, ids, gain=w[0, :1]), lambda: hif4.hif4_combine(x, ids, w[:, :1]),
              lambda: hif4.hif4_combine(x, ids, residual=x[:3]), lambda: hif4.hif4_combine_backward(x, ids, w, want_dweights=True),
              lambda: hif4.hif4_route_backward(w[:3], x, ids), lambda: hif4.hif4_combine(x, ids, residual=x, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: hif4.hif4_route(x.double(), 2), lambda: hif4.hif4_route(None, 2), lambda: hif4.hif4_combine(x.int(), ids)):
        with pytest.raises(TypeError):
            f()
    assert hif4.launch_count() == before


@pytest.mark.parametrize("T", [1, 20, 300])
@pytest.mark.parametrize("fmt", ["hif4", "mxfp4", "nvfp4"])
def test_a_layer_of_experts_together(hif4, T, fmt):
    """Routing, rows, two grouped products around an activation, combination: against the same steps in 64 bits on the operands as
    converted."""
    g = gen(T)
    E, k, K, N = 12, 3, 256, 128
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    x, up, down = rnd(T, K), rnd(E * 2 * N, K) / 16, rnd(E * K, N) / 8
    logits, res = torch.randn(T, E, generator=g, device="cuda"), rnd(T, K)
    logits[T // 2] = -math.inf                                    # a padded token reaches no expert
    ids, w = hif4.hif4_route(logits, k, score=SIGMOID, scale=2.0)
    off, row_of = hif4.hif4_expert_plan(ids, E)
    code = {"hif4": 0, "mxfp4": 1, "nvfp4": 2}[fmt]
    used = int(off[-1])
    if fmt == "hif4":
        q = lambda v: hif4.hif4_quantize(v)      # noqa: E731
        wu, wd = q(up).view(E, 2 * N, K // 64, 36), q(down).view(E, K, N // 64, 36)
        values = lambda u: hif4.hif4_dequantize(u, torch.float32).double()      # noqa: E731
        product = lambda a, b: hif4.hif4_grouped_gemm(a[:used], b, off)         # noqa: E731
    else:
        q = lambda v: hif4.hif4_bfp4_quantize(v, code)      # noqa: E731

        def grouped(v, rows):
            c, s = q(v)
            return c.view(E, rows, -1), s.view(s.shape[0], E, rows, 16).transpose(0, 1).contiguous()
        wu, wd = grouped(up, 2 * N), grouped(down, K)
        values = lambda u: ref.values(*u, code)      # noqa: E731
        product = lambda a, b: hif4.hif4_bfp4_grouped_gemm(a, b, off, code, dtype=torch.float32)      # noqa: E731
    rows = hif4.hif4_dispatch(x, row_of, fmt=code)
    h = product(rows, wu)
    act = (torch.nn.functional.silu(h[:used, :N]) * h[:used, N:]).to(torch.bfloat16)
    y = hif4.hif4_combine(product(q(act), wd), row_of, w, residual=res)
    X, U, D = values(q(x)), values(q(up)).view(E, 2 * N, K), values(q(down)).view(E, K, N)
    A = values(q(act))
    want, size = res.double(), res.double().abs()
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            if e < 0:
                continue
            r = int(row_of[t, j])
            z = U[e] @ X[t]
            assert torch.allclose(h[r].double(), z, rtol=0, atol=1e-5 * float((U[e].abs() @ X[t].abs()).max()))
            want[t] += float(w[t, j]) * (D[e] @ A[r])
            size[t] += abs(float(w[t, j])) * (D[e].abs() @ A[r].abs())
    assert bool(((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2e-5 * size).all())
    if T > 1:
        assert torch.equal(y[T // 2], res[T // 2])


def test_a_layer_in_a_graph_on_another_stream(hif4):
    """Captured once, replayed with other inputs: nothing is kept from the call that was captured."""
    E, k, K, N = 16, 4, 512, 256
    x, logits = torch.randn(100, K, device="cuda").to(torch.bfloat16), torch.randn(100, E, device="cuda")
    c, s = hif4.hif4_bfp4_quantize((torch.randn(E * N, K, device="cuda") / 16).to(torch.bfloat16), 2)
    b = c.view(E, N, -1), s.view(-1, E, N, 16).transpose(0, 1).contiguous()

    def layer(x, logits):
        ids, w = hif4.hif4_route(logits, k)
        off, row_of = hif4.hif4_expert_plan(ids, E)
        return hif4.hif4_combine(hif4.hif4_bfp4_grouped_gemm(hif4.hif4_dispatch(x, row_of, fmt=2), b, off, 2, dtype=torch.float32), row_of, w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, logits)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = layer(x, logits)
    torch.cuda.current_stream().wait_stream(side)
    for seed in range(3):
        x.copy_(torch.randn(100, K, generator=gen(seed), device="cuda"))
        logits.copy_(torch.randn(100, E, generator=gen(seed + 9), device="cuda"))
        graph.replay()
        assert torch.equal(y, layer(x, logits))


@pytest.mark.parametrize("T", [1, 150])
@pytest.mark.parametrize("fmt", [1, 2])
def test_training_step_of_a_layer(hif4, T, fmt):
    """Forward and backward of routing, rows, grouped product and combination, every gradient call fed by the one before: against the
    formulas in 64 bits on the operands as converted.  (Conversions are passed straight through.)"""
    g = gen(T + fmt)
    E, k, K, N = 10, 2, 192, 256
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    x, w, dout, logits = rnd(T, K), rnd(E * N, K) / 8, rnd(T, N), torch.randn(T, E, generator=g, device="cuda")
    V = lambda q: ref.values(*q, fmt)      # noqa: E731

    def grouped(v, rows):
        c, s = hif4.hif4_bfp4_quantize(v.contiguous(), fmt)
        return c.view(E, rows, -1), s.view(s.shape[0], E, rows, 16).transpose(0, 1).contiguous()
    weights = grouped(w, N)                                              # laid out once: rows for the product, columns for its gradient
    turned = [hif4.hif4_bfp4_quantize_transposed(e, fmt) for e in w.view(E, N, K)]
    columns = torch.stack([c for c, _ in turned]), torch.stack([s for _, s in turned])
    ids, p = hif4.hif4_route(logits, k)
    off, row_of = hif4.hif4_expert_plan(ids, E)
    rows = hif4.hif4_dispatch(x, row_of, fmt=fmt)
    y = hif4.hif4_bfp4_grouped_gemm(rows, weights, off, fmt, dtype=torch.float32)
    out = hif4.hif4_combine(y, row_of, p, dtype=torch.bfloat16)
    dy, dp = hif4.hif4_combine_backward(dout, row_of, p, rows=y)
    drows = hif4.hif4_bfp4_grouped_gemm(hif4.hif4_bfp4_quantize(dy, fmt), columns, off, fmt, dtype=torch.float32)
    dx = hif4.hif4_combine(drows, row_of, dtype=torch.bfloat16)
    dlogits = hif4.hif4_route_backward(dp, logits, ids)
    # the same with the converted operands
    X, W, WT = V(hif4.hif4_bfp4_quantize(x, fmt)), V(weights), V(columns).transpose(1, 2)
    at = ids.long()
    l64 = logits.double().requires_grad_()
    P = torch.softmax(l64.gather(1, at), 1)
    Y = torch.einsum("tkno,to->tkn", W[at], X)
    dY = V(hif4.hif4_bfp4_quantize(dy, fmt))[row_of.long()]
    want = {"out": (P.unsqueeze(-1) * Y).sum(1), "dp": (dout.double().unsqueeze(1) * Y).sum(-1),
            "dx": torch.einsum("tkn,tkno->to", dY, WT[at])}
    want["dlogits"], = torch.autograd.grad(P, l64, want["dp"].detach())
    size = {"out": (Y.abs()).sum(1), "dp": (dout.double().abs().unsqueeze(1) * Y.abs()).sum(-1), "dx": torch.einsum("tkn,tkno->to", dY.abs(), WT[at].abs())}
    size["dlogits"] = size["dp"].amax(1, keepdim=True)
    for name, got, roundings in (("out", out, 2.0 ** -8), ("dp", dp, 0.0), ("dx", dx, 2.0 ** -8), ("dlogits", dlogits, 0.0)):
        ref64 = want[name].detach()
        # a product's FP32 sums: 1e-5 of the terms; the combinations after it add fewer; one rounding to BF16
        assert bool(((got.double() - ref64).abs() <= roundings * ref64.abs() + 3e-5 * size[name].detach()).all()), name
    # rounded to the type of the experts' rows (FP32): the weight times the token's gradient
    assert torch.equal(dy[row_of.long()], p.unsqueeze(-1) * dout.float().unsqueeze(1))


def test_plan_workspaces(hif4):
    ids = torch.randint(0, 64, (3000, 2), device="cuda", dtype=torch.int32)
    need = hif4.hif4_expert_plan_workspace(3000, 2, 64)
    want = hif4.hif4_expert_plan(ids, 64)
    got = hif4.hif4_expert_plan(ids, 64, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert need > 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for space, code in ((torch.empty(need - 1, dtype=torch.uint8, device="cuda"), 5), (torch.empty(need + 64, dtype=torch.uint8, device="cuda")[64:], 3)):
        with pytest.raises(hif4.Hif4Error) as e:
            hif4.hif4_expert_plan(ids, 64, workspace=space)
        assert e.value.code == code
    with pytest.raises(ValueError):
        hif4.hif4_expert_plan(ids, 64, workspace=torch.empty(1, dtype=torch.uint8, device="cuda").expand(need))


def test_calls_on_a_stream_of_their_own(hif4):
    """stream=: the call and its allocations belong to that stream; two streams at once keep out of each other's way."""
    x, logits = torch.randn(500, 256, device="cuda").to(torch.bfloat16), torch.randn(500, 40, device="cuda")
    c, s = hif4.hif4_bfp4_quantize(torch.randn(40 * 128, 256, device="cuda").to(torch.bfloat16), 2)
    b = c.view(40, 128, -1), s.view(-1, 40, 128, 16).transpose(0, 1).contiguous()

    def layer(st):
        ids, w = hif4.hif4_route(logits, 6, stream=st)
        off, row_of = hif4.hif4_expert_plan(ids, 40, stream=st)
        rows = hif4.hif4_dispatch(x, row_of, fmt=2, stream=st)
        y = hif4.hif4_bfp4_grouped_gemm(rows, b, off, 2, stream=st)
        return hif4.hif4_combine(y, row_of, w, stream=st)
    want = layer(None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [layer(st) for _ in range(4) for st in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(v, want) for v in got)
