"""hif4_linear_act, hif4_gated_linear and their gradients at the edges of their arguments: a single row with any stride,
infinite and NaN gradients, more rows than a grid has blocks, activations without the slack of a product, captured graphs.

Tolerances as in test_gpu_linear_act.py; an activation alone is within (8 + 2 |e|) 2^-22 of its value, e the exponent that its
formula has (-z, z^2 / 2, or twice the argument of tanh): two units of 2^-23 for each of the exponential, the division and the
roundings around them, and e times the rounding of the exponent itself.  A sigmoid below 2^-126 is zero."""
import pytest
import torch

from tests.test_gpu_linear_act import FN, TINY, TOL, TYPES, U, act64, call, close, decode, expect_forward, hif4, operands, products64  # noqa: F401

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


# ------------------------------------------------------------------------------------------------------ NaN and infinity
def nonzero_weights(hif4, N, K, seed):
    """Codes without a zero: the product with an infinity is an infinity of the weight's sign."""
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    w = hif4.hif4_quantize(torch.where(torch.rand(N, K, generator=g, device="cuda") < 0.5, -1.0, 1.0).to(torch.bfloat16))
    assert bool((decode(hif4, w) != 0).all())
    return w


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_an_infinite_gradient_stays_infinite(hif4, dtype, act, M):
    """dX[m] = sum of dZ[m, n] W[n]: one infinite dZ and no zero among the codes give infinities, not NaN, in that row alone."""
    N, K = 192, 512
    x, _, b = operands(hif4, M, 1, K, dtype, False, 3)
    w = nonzero_weights(hif4, N, K, 4)
    bias = torch.full((N,), 3.0, dtype=dtype, device="cuda")
    dy = torch.randn(M, N, device="cuda").to(dtype)
    clean, dbc = hif4.hif4_linear_act_backward(dy, x, w, bias, act=act, want_dbias=True)
    n, m = 77, M // 2
    if act:            # an output whose slope is positive
        z = decode(hif4, hif4.hif4_quantize(x)) @ decode(hif4, w).t() + 3.0
        n = int(z[m].argmax())
        assert float(z[m, n]) > 1.0
    dy[m, n] = float("inf")
    dx, db = hif4.hif4_linear_act_backward(dy, x, w, bias, act=act, want_dbias=True)
    want = decode(hif4, w)[n].sign() * float("inf")
    assert torch.equal(dx[m].double(), want)
    keep = torch.arange(M, device="cuda") != m
    assert torch.equal(dx[keep], clean[keep])
    keep = torch.arange(N, device="cuda") != n
    assert torch.equal(db[keep], dbc[keep]) and float(db[n]) == float("inf")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [3, 300])
def test_a_nan_gradient_stays_in_its_row_and_column(hif4, gated, dtype, M):
    x, w, b = operands(hif4, M, 256, 512, dtype, gated, 5)
    dy = torch.randn(M, 256, device="cuda").to(dtype)
    f = hif4.hif4_gated_linear_backward if gated else hif4.hif4_linear_act_backward
    clean = f(dy, x, *w, *b, act=3, want_dbias=True)
    dy[1, 9] = float("nan")
    got = f(dy, x, *w, *b, act=3, want_dbias=True)
    assert torch.isnan(got[0][1]).all()
    rows = torch.arange(M, device="cuda") != 1
    cols = torch.arange(256, device="cuda") != 9
    assert torch.equal(got[0][rows], clean[0][rows])
    for g, c in zip(got[1:], clean[1:]):
        assert torch.isnan(g[9]) and torch.equal(g[cols], c[cols])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [1, 12, 40, 300])
def test_infinite_activations_residuals_and_results(hif4, M, gated):
    """An infinite activation saturates in the conversion; an infinite residual and a result past FP16's range are infinities."""
    x, w, b = operands(hif4, M, 256, 512, torch.float16, gated, 6)
    x[0, 3], x[-1, 200] = float("inf"), float("-inf")
    res = torch.randn(M, 256, device="cuda").to(torch.float16)
    res[0, 5], res[-1, 6] = float("inf"), float("-inf")
    res[-1, 7] = 60000.0
    y = call(hif4, x, w, b, act=1, residual=res, res_scale=2.0)
    ref, e = expect_forward(hif4, x, w, b, 1, res, 2.0)
    e = torch.where(torch.isinf(ref), torch.zeros_like(e), e)
    over = ref.abs() - e > 65520.0
    under = ref.abs() + e < 65520.0
    assert bool(over[0, 5]) and bool(over[-1, 6]) and bool(over[-1, 7])
    assert torch.equal(y[over].double(), ref[over].sign() * float("inf"))
    close(y[under], ref[under], e[under], torch.float16, "finite results")
    u = call(hif4, x, w, b, act=1, residual=res, res_scale=2.0, units=True, dtype=torch.float16)
    assert torch.equal(u, hif4.hif4_quantize(y))


# -------------------------------------------------------------------------------------------------- rows past 65535 x 32
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradient_without_activation_of_two_million_rows(hif4, dtype):
    M, N, K = 65535 * 32 + 33, 8, 64
    _, w, _ = operands(hif4, 1, N, K, dtype, False, 3)
    dy = torch.randn(M, N, device="cuda").to(dtype)
    dx, db = hif4.hif4_linear_act_backward(dy, None, w[0], want_dbias=True)
    wd = decode(hif4, w[0])
    for r in range(0, M, 1 << 19):
        d = dy[r:r + (1 << 19)].double()
        close(dx[r:r + (1 << 19)], d @ wd, (TOL + 2.0 ** -16) * (d.abs() @ wd.abs()), dtype, f"dx from {r}")
    # 32 rows in series, then 2049 row blocks for each of 32 ways, then the ways
    close(db, dy.double().sum(0), 2.0 ** -24 * (32 + 2049 + 32) * dy.double().abs().sum(0), torch.float32, "dbias")


# ----------------------------------------------------------------------------------------------------- activations alone
def exponent(z, act):
    if act == 2:
        return z.abs()
    if act == 3:
        return z * z / 2
    if act == 4:
        return (2 * (2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)).abs()
    return torch.zeros_like(z)


def value_and_slope64(z, act):
    """The tanh form as z times a sigmoid of 2u: 1 + tanh(u) and 1 - tanh(u)^2 cancel in the left tail, in 64 bits too."""
    if act != 4:
        return act64(z, act)
    c = 2 * (2 / torch.pi) ** 0.5
    s = torch.sigmoid(c * (z + 0.044715 * z ** 3))
    r = torch.sigmoid(-c * (z + 0.044715 * z ** 3))
    return z * s, s + z * s * r * c * (1 + 3 * 0.044715 * z * z)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 256), (40, 256), (2, 0)])
def test_activation_of_a_bias(hif4, act, gated, dtype, M, K):
    """Zero activations leave act(bias) alone, from the streaming form, the tensor-core form and without a contraction."""
    N = 1024
    x, w, _ = operands(hif4, M, N, 256, dtype, gated, 2)
    b = [torch.linspace(-12.0, 12.0, N, device="cuda").to(dtype), torch.full((N,), 3.0, dtype=dtype, device="cuda")][:len(w)]
    y = call(hif4, torch.zeros_like(x)[:, :K].contiguous(), [t[:, :K // 64].contiguous() for t in w], b, act=act)
    z = b[0].double()
    a, _ = value_and_slope64(z, act)
    up = 3.0 if gated else 1.0
    err = up * ((8 + 2 * exponent(z, act)) * 2.0 ** -22 * a.abs() + z.abs() * 2.0 ** -126)
    close(y, (up * a).expand(M, N), err.expand(M, N), dtype, f"act {act}")


@pytest.mark.parametrize("act", range(1, 5))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_slope_at_a_bias(hif4, act, dtype):
    """One row of gradients of one: the bias gradient is act'(bias) in FP32.  Its two terms, the value's factor f and z f', carry the
    activation's relative error each; for a sigmoid f of exponent e(z), z f' = z e' f (1 - f), so a sigmoid that is zero below 2^-126
    leaves out up to (1 + |z e'|) 2^-126."""
    N, K = 1024, 256
    x, w, _ = operands(hif4, 1, N, K, dtype, False, 2)
    b = torch.linspace(-12.0, 12.0, N, device="cuda").to(dtype)
    _, db = hif4.hif4_linear_act_backward(torch.ones(1, N, dtype=dtype, device="cuda"), torch.zeros_like(x), w[0], b, act=act, want_dx=False, want_dbias=True)
    z = b.double()
    a, s = value_and_slope64(z, act)
    rate = 2 * (2 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z) if act == 4 else 1.0
    first = torch.where(z == 0, torch.full_like(z, 0.5), a / torch.where(z == 0, torch.ones_like(z), z)).abs()
    err = (8 + 2 * exponent(z, act)) * 2.0 ** -22 * (first + (s - first).abs()) + 2.0 ** -22 * first * z.abs() + (1 + z.abs() * rate) * 2.0 ** -126
    close(db, s, err, torch.float32, f"slope {act}")


# ------------------------------------------------------------------------------------------------------- captured graphs
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(64, 512, 8192), (300, 4096, 1024), (2000, 2300, 512)])
def test_pair_kernels_in_a_graph(hif4, M, N, K, gated):
    """K slices, whole rounds and balanced rounds: the counts of finished parts are cleared by every replay."""
    x, w, b = operands(hif4, M, N, K, torch.bfloat16, gated, 8)
    dy = torch.randn(M, N, device="cuda").to(torch.bfloat16)
    back = hif4.hif4_gated_linear_backward if gated else hif4.hif4_linear_act_backward
    want, dwant = call(hif4, x, w, b, act=2), back(dy, x, *w, *b, act=2, want_dbias=True)
    out = torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(hif4, x, w, b, act=2, out=out)
        back(dy, x, *w, *b, act=2, want_dbias=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(hif4, x, w, b, act=2, out=out)
        grads = back(dy, x, *w, *b, act=2, want_dbias=True)
    for _ in range(3):
        out.zero_()
        for t in grads:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(g, v) for g, v in zip(grads, dwant))
    assert hif4.hif4_last_device_status() == 0


# ---------------------------------------------------------------------------------------------- dZ as one or two numbers
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("M,N,K", [(1, 64, 256), (40, 1000, 320), (300, 513, 512), (130, 4096, 256)])
def test_precise_gradient(hif4, gated, act, M, N, K):
    """BF16 with dZ in two parts: 2^-16 of it in the product's error where one part leaves 2^-8; bias gradients keep their bits."""
    x, w, b = operands(hif4, M, N, K, torch.bfloat16, gated, M + N)
    dy = torch.randn(M, N, device="cuda").to(torch.bfloat16)
    f = hif4.hif4_gated_linear_backward if gated else hif4.hif4_linear_act_backward
    one, two, again = (f(dy, x, *w, *b, act=act, want_dbias=True, precise=p) for p in (False, True, True))
    assert all(torch.equal(a, v) for a, v in zip(two, again)) and all(torch.equal(a, v) for a, v in zip(one[1:], two[1:]))
    p = products64(hif4, x, w, b)
    z, ez, wg = p[0]
    a, s = act64(z, act)
    D = dy.double()
    es = 2 * ez + FN * (s.abs() + z.abs()) if act else torch.zeros_like(z)
    if act == 1:
        es = es + (z.abs() <= ez).double()                    # the step at zero
    if gated:
        u, eu, wu = p[1]
        grads = [(D * u * s, D.abs() * (es * (u.abs() + eu) + s.abs() * eu), wg), (D * a, D.abs() * (1.2 * ez + FN * a.abs()), wu)]
    else:
        grads = [(D * s, D.abs() * es, wg)]
    ref = sum(dz @ wd for dz, _, wd in grads)
    err = sum((e + (2.0 ** -16 + TOL) * dz.abs()) @ wd.abs() for dz, e, wd in grads)
    close(two[0], ref, err, torch.bfloat16, "dx")
    if gated or act > 1:                                      # else dZ is dY or zero: one BF16 number holds it
        assert float((two[0].double() - ref).norm()) <= float((one[0].double() - ref).norm())
