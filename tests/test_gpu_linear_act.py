"""hif4_linear_act, hif4_gated_linear and their gradients against the formulas in 64 bits on the decoded operands.

Tolerances.  A product is within 1e-5 * sum |a||b| of the exact one (the GEMM's tolerance); an activation has a slope of at
most 1.2 and is computed to 2^-18 of its size (FP32 exp, division, erfc and a handful of roundings, exponents up to 88); a
result is rounded once to its type (relative 2^-8 BF16, 2^-11 FP16, 2^-24 FP32).  Gradients: act' has a slope of at most 2;
dZ goes into the last product as one BF16 number (2^-8) for BF16, two (2^-16) for FP16."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}
TOL, FN = 1e-5, 2.0 ** -18
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def hif4():
    assert torch.cuda.is_available()
    import paper_2602_11287_b200 as lib
    return lib


def act64(z, act):
    if act == 1:
        return z.clamp(min=0), (z > 0).double()
    if act == 2:
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if act == 3:
        phi = 0.5 * torch.erfc(-z / 2 ** 0.5)
        return z * phi, phi + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    if act == 4:
        c = (2 / torch.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return z, torch.ones_like(z)


def operands(hif4, M, N, K, dtype, gated, seed, bias=True, std=1.0):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")       # noqa: E731
    x = (rnd(M, K) * std).to(dtype)
    w = [hif4.hif4_quantize((rnd(N, K) * 1.5 / max(K, 1) ** 0.5).to(torch.bfloat16)) for _ in range(2 if gated else 1)]
    b = [rnd(N).to(dtype) if bias else None for _ in w]
    return x, w, b


def decode(hif4, units):
    return hif4.hif4_dequantize(units, torch.float32).double() if units.numel() else torch.zeros(units.shape[0], units.shape[1] * 64, dtype=torch.float64, device="cuda")


def products64(hif4, x, w, b, mode=0):
    xq = decode(hif4, x if x.dtype == torch.uint8 else hif4.hif4_quantize(x, mode=mode)) if (x.shape[1] if x.dim() == 2 else 1) else x.double()
    out = []
    for wi, bi in zip(w, b):
        wd = decode(hif4, wi)
        z = xq @ wd.t()
        e = TOL * (xq.abs() @ wd.abs().t())
        if bi is not None:
            z = z + bi.double()
            e = e + FN * bi.double().abs()
        out.append((z, e, wd))
    return out


def close(got, ref, err, dtype, what):
    d = (got.double() - ref).abs()
    bound = U[dtype] * ref.abs() + err + TINY[dtype]
    assert not torch.isnan(got.double()).any(), what
    worst = float((d / bound).max()) if d.numel() else 0.0
    assert worst <= 1.0, f"{what}: worst ratio {worst:.3g}"


def expect_forward(hif4, x, w, b, act, res, scale, mode=0):
    p = products64(hif4, x, w, b, mode)
    z, ez, _ = p[0]
    a, _ = act64(z, act)
    ea = 1.2 * ez + FN * a.abs()
    if len(w) == 2:
        u, eu, _ = p[1]
        y, e = a * u, ea * (u.abs() + eu) + a.abs() * eu
    else:
        y, e = a, ea
    if res is not None:
        y = y + scale * res.double()
        e = e + FN * (scale * res.double()).abs()
    return y, e


def call(hif4, x, w, b, **kw):
    if len(w) == 2:
        return hif4.hif4_gated_linear(x, w[0], w[1], b[0], b[1], **kw)
    return hif4.hif4_linear_act(x, w[0], b[0], **kw)


SHAPES = [(1, 1, 64), (1, 64, 64), (2, 70, 128), (1, 1000, 256), (3, 333, 512), (8, 256, 1024), (9, 129, 256), (16, 1024, 768), (17, 40, 256),
          (31, 200, 320), (32, 513, 512), (33, 300, 256), (64, 2049, 448), (77, 1001, 1024), (128, 128, 256), (129, 129, 64), (200, 260, 704),
          (257, 513, 256), (300, 1, 512), (513, 1000, 1280)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_forward_sizes(hif4, M, N, K, gated):
    for n, dtype in enumerate(TYPES):
        act = (M + N + n) % 5
        x, w, b = operands(hif4, M, N, K, dtype, gated, M * 3 + N + K, bias=n != 1)
        res = torch.randn(M, N, device="cuda").to(dtype) if n != 2 else None
        y = call(hif4, x, w, b, act=act, residual=res, res_scale=0.5)
        ref, e = expect_forward(hif4, x, w, b, act, res, 0.5)
        close(y, ref, e, dtype, f"{M}x{N}x{K} {dtype} act {act}")
        assert torch.equal(y, call(hif4, x, w, b, act=act, residual=res, res_scale=0.5)), "two runs differ"
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 14336, 4096), (4, 4096, 14336), (16, 5120, 5120), (64, 4096, 4096), (256, 512, 8192), (100, 1024, 14336),
                                   (700, 4000, 2048), (1500, 5120, 1024), (2048, 1024, 4160), (4096, 2100, 512)])
def test_forward_large(hif4, M, N, K, gated):
    """Long contractions (tiles shared along K), several rounds of tiles, partial last rounds."""
    x, w, b = operands(hif4, M, N, K, torch.bfloat16, gated, M + N)
    res = torch.randn(M, N, device="cuda").to(torch.bfloat16)
    y = call(hif4, x, w, b, act=2, residual=res, res_scale=-0.25)
    ref, e = expect_forward(hif4, x, w, b, 2, res, -0.25)
    close(y, ref, e, torch.bfloat16, f"{M}x{N}x{K}")
    assert torch.equal(y, call(hif4, x, w, b, act=2, residual=res, res_scale=-0.25)), "two runs differ"
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [5, 150])
def test_activations_over_their_range(hif4, act, gated, M):
    """Products from near zero to the far tails of exp and erfc."""
    x, w, b = operands(hif4, M, 192, 256, torch.float32, gated, 77 + act, std=1.0)
    x = x * torch.logspace(-3, 2.3, M, device="cuda").unsqueeze(1)
    y = call(hif4, x, w, b, act=act)
    ref, e = expect_forward(hif4, x, w, b, act, None, 0.0)
    close(y, ref, e, torch.float32, f"act {act}")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 64, 256), (7, 192, 512), (30, 1024, 320), (40, 128, 256), (130, 320, 512), (300, 4096, 256)])
@pytest.mark.parametrize("mode", [0, 1])
def test_units_in_and_out(hif4, dtype, M, N, K, gated, mode):
    x, w, b = operands(hif4, M, N, K, dtype, gated, M + K)
    res = torch.randn(M, N, device="cuda").to(dtype)
    y = call(hif4, x, w, b, act=2, residual=res, mode=mode)
    xu = hif4.hif4_quantize(x, mode=mode)
    assert torch.equal(call(hif4, xu, w, b, act=2, residual=res, dtype=dtype, mode=mode), y)
    u = call(hif4, x, w, b, act=2, residual=res, units=True, dtype=dtype, mode=mode)
    assert torch.equal(u, hif4.hif4_quantize(y, mode=mode))
    ref, e = expect_forward(hif4, x, w, b, 2, res, 1.0, mode)
    close(y, ref, e, dtype, "y")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(3, 77, 256), (20, 100, 320), (50, 200, 256), (200, 300, 512)])
@pytest.mark.parametrize("pad,off", [(16, 8), (13, 0), (8, 1), (7, 3)])
def test_strides_guards_and_in_place_residual(hif4, dtype, M, N, K, gated, pad, off):
    x, w, b = operands(hif4, M, N, K, dtype, gated, M + K + pad)
    wide = torch.zeros(M, K + 64, dtype=dtype, device="cuda")
    wide[:, 16:16 + K] = x
    res = torch.randn(M, N, device="cuda").to(dtype)
    buf = torch.full((M + 2, N + pad + off), 9.0, dtype=dtype, device="cuda")
    out = buf[1:M + 1, off:off + N]
    out.copy_(res)
    y = call(hif4, wide[:, 16:16 + K], w, b, act=3, residual=out, res_scale=2.0, out=out)
    assert y is out
    ref, e = expect_forward(hif4, x, w, b, 3, res, 2.0)
    close(y, ref, e, dtype, "strided")
    assert torch.equal(y.contiguous(), call(hif4, x, w, b, act=3, residual=res, res_scale=2.0))
    out.fill_(9.0)
    assert (buf == 9.0).all(), "written outside the matrix"


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [1, 20, 40, 200])
def test_weights_at_any_unit_address(hif4, M, gated):
    """Weights that start four bytes off a 16-byte boundary (a slice of a packed file)."""
    x, w, b = operands(hif4, M, 96, 512, torch.bfloat16, gated, M)
    y = call(hif4, x, w, b, act=2)
    moved = []
    for wi in w:
        flat = torch.empty(wi.numel() + 16, dtype=torch.uint8, device="cuda")
        v = flat[4:4 + wi.numel()].view(wi.shape)
        v.copy_(wi)
        moved.append(v)
    got = call(hif4, x, moved, b, act=2)
    ref, e = expect_forward(hif4, x, w, b, 2, None, 0.0)
    close(got, ref, e, torch.bfloat16, "moved weights")
    close(y, ref, e, torch.bfloat16, "weights")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [1, 12, 40, 300])
def test_nan_and_infinity(hif4, M, gated):
    """A NaN activation makes its row NaN, a NaN weight unit its column; nothing else changes."""
    x, w, b = operands(hif4, M, 256, 512, torch.bfloat16, gated, 5)
    clean = call(hif4, x, w, b, act=2)
    x[0, 100] = float("nan")
    w[-1][7, 3, 0] = 0xFF
    y = call(hif4, x, w, b, act=2)
    assert torch.isnan(y[0]).all() and torch.isnan(y[:, 7]).all()
    keep = torch.ones(256, dtype=torch.bool, device="cuda"); keep[7] = False
    assert torch.equal(y[1:, keep], clean[1:, keep])
    u = call(hif4, x, w, b, act=2, units=True, dtype=torch.bfloat16)
    assert torch.equal(u, hif4.hif4_quantize(y))


def test_empty_sizes_and_k_zero(hif4):
    x, w, b = operands(hif4, 4, 64, 256, torch.bfloat16, True, 1)
    assert hif4.hif4_linear_act(x[:0], w[0], b[0]).shape == (0, 64)
    y = hif4.hif4_gated_linear(x[:, :0], w[0][:, :0], w[1][:, :0], b[0], b[1], act=2)          # no contraction: the biases alone
    a, _ = act64(b[0].double(), 2)
    close(y, (a * b[1].double()).expand(4, 64), (FN * a * b[1].double()).abs().expand(4, 64), torch.bfloat16, "K = 0")
    dx, db = hif4.hif4_linear_act_backward(y[:0], x[:0], w[0], act=2, want_dbias=True)
    assert dx.shape == (0, 256) and (db == 0).all()


def test_other_stream(hif4):
    x, w, b = operands(hif4, 300, 2048, 1024, torch.bfloat16, True, 8)
    want = call(hif4, x, w, b)
    dwant = hif4.hif4_gated_linear_backward(want, x, w[0], w[1])[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(10):
        outs.append((call(hif4, x, w, b, stream=s), hif4.hif4_gated_linear_backward(want, x, w[0], w[1], stream=s)[0]))
        for n in (1 << 20, 1 << 23, 1 << 24):
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    for y, d in outs:
        assert torch.equal(y, want) and torch.equal(d, dwant)


def test_in_a_graph(hif4):
    x, w, b = operands(hif4, 3, 512, 1024, torch.bfloat16, True, 8)
    want = call(hif4, x, w, b)
    out = torch.empty_like(want)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(hif4, x, w, b, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(hif4, x, w, b, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------------------------ gradients
def check_backward(hif4, M, N, K, dtype, gated, act, bias=True, strided=False):
    x, w, b = operands(hif4, M, N, K, dtype, gated, M + 2 * N + K, bias=bias)
    dy = torch.randn(M, N, device="cuda").to(dtype)
    if strided:
        wide = torch.zeros(M, N + 5, dtype=dtype, device="cuda")
        wide[:, 3:3 + N] = dy
        dy = wide[:, 3:3 + N]
    if gated:
        dx, db, dbu = hif4.hif4_gated_linear_backward(dy, x, w[0], w[1], b[0], b[1], act=act, want_dbias=True)
        again = hif4.hif4_gated_linear_backward(dy, x, w[0], w[1], b[0], b[1], act=act, want_dbias=True)
    else:
        dx, db = hif4.hif4_linear_act_backward(dy, x, w[0], b[0], act=act, want_dbias=True)
        again = hif4.hif4_linear_act_backward(dy, x, w[0], b[0], act=act, want_dbias=True)
    assert torch.equal(dx, again[0]) and torch.equal(db, again[1]), "two runs differ"
    p = products64(hif4, x, w, b)
    D = dy.double()
    z, ez, wg = p[0]
    a, s = act64(z, act)
    es = 2 * ez + FN * (s.abs() + z.abs()) if act else torch.zeros_like(z)
    if act == 1:
        es = es + (z.abs() <= ez).double()                    # the step at zero
    if gated:
        u, eu, wu = p[1]
        grads = [(D * u * s, D.abs() * (es * (u.abs() + eu) + s.abs() * eu), wg), (D * a, D.abs() * (1.2 * ez + FN * a.abs()), wu)]
    else:
        grads = [(D * s, D.abs() * es, wg)]
    part = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -16
    ref, err = 0, 0
    for dz, e, wd in grads:
        ref = ref + dz @ wd
        err = err + (e + (part + TOL) * dz.abs()) @ wd.abs()
    close(dx, ref, err, dtype, f"dx {M}x{N}x{K}")
    for got, (dz, e, _) in zip((db, dbu) if gated else (db,), grads):
        close(got, dz.sum(0), (e + 2.0 ** -24 * (64 + M / 32) * dz.abs() + FN * dz.abs()).sum(0), torch.float32, "dbias")
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 1, 64), (1, 64, 256), (3, 70, 192), (8, 300, 512), (33, 129, 256), (40, 1000, 320), (129, 257, 576),
                                   (300, 64, 1024), (257, 512, 256), (600, 1100, 768)])
def test_gradient_sizes(hif4, M, N, K, gated, dtype):
    check_backward(hif4, M, N, K, dtype, gated, act=(M + N) % 5, bias=M % 2 == 0, strided=N % 2 == 0)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(2, 14336, 1024), (64, 8192, 512), (300, 4096, 4096), (1024, 1536, 2048), (2000, 700, 1536)])
def test_gradient_large(hif4, M, N, K, gated):
    check_backward(hif4, M, N, K, torch.bfloat16, gated, act=2)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(2860, 15, 6144), (806, 36, 12032), (2507, 78, 7424), (936, 64, 12416), (1200, 130, 8192)])
def test_gradient_of_many_tiles_with_a_short_contraction(hif4, M, N, K, gated):
    """Each CTA pair works through several tiles of one to four contraction steps: the decode warps that join the epilogue
    of the last tile must not take an earlier tile's completion for its own."""
    for dtype in (torch.bfloat16, torch.float16):
        check_backward(hif4, M, N, K, dtype, gated, act=2)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(3000, 4000, 64), (2000, 9000, 128), (5000, 2049, 256)])
def test_forward_of_many_tiles_with_a_short_contraction(hif4, M, N, K, gated):
    x, w, b = operands(hif4, M, N, K, torch.bfloat16, gated, M + N)
    y = call(hif4, x, w, b, act=2)
    ref, e = expect_forward(hif4, x, w, b, 2, None, 0.0)
    close(y, ref, e, torch.bfloat16, f"{M}x{N}x{K}")
    for _ in range(3):
        assert torch.equal(y, call(hif4, x, w, b, act=2)), "two runs differ"


@pytest.mark.parametrize("act", range(5))
def test_gradient_activations(hif4, act):
    for gated in (False, True):
        check_backward(hif4, 200, 192, 256, torch.float16, gated, act)


@pytest.mark.parametrize("act", [2, 3, 4])
@pytest.mark.parametrize("gated", [False, True])
def test_bias_gradient_against_differences(hif4, act, gated):
    """d/db of sum(y * c) by centred differences of the FP32 forward call (bias in FP32); the gradient call takes the same
    bias and c, representable in BF16.  Step 2^-4: third derivatives of the activations stay below 2, so the difference is within
    2/6 * 2^-8 of the slope, and 1e-5 / 2^-4 of the product's rounding."""
    M, N, K = 20, 64, 256
    x, w, b = operands(hif4, M, N, K, torch.bfloat16, gated, 3)
    c = torch.randn(M, N, device="cuda").to(torch.bfloat16)
    if gated:
        _, db, dbu = hif4.hif4_gated_linear_backward(c, x, w[0], w[1], b[0], b[1], act=act, want_dx=False, want_dbias=True)
    else:
        _, db = hif4.hif4_linear_act_backward(c, x, w[0], b[0], act=act, want_dx=False, want_dbias=True)
    e = 2.0 ** -4
    for i, got in enumerate((db, dbu) if gated else (db,)):
        up, down = ([bj.float() + (s * e if j == i else 0.0) for j, bj in enumerate(b)] for s in (1, -1))
        fu, fd = (call(hif4, x, w, bb, act=act, dtype=torch.float32).double() for bb in (up, down))
        diff = ((fu - fd) * c.double()).sum(0) / (2 * e)
        p = products64(hif4, x, w, b)
        size = (c.double().abs() * (p[1][0].abs() if gated and i == 0 else 1.0)).sum(0) + 1.0
        assert ((diff - got.double()).abs() <= (2 / 6 * 2.0 ** -8 + 1e-3) * size).all()


def test_gradients_that_are_not_wanted_and_without_activation(hif4):
    x, w, b = operands(hif4, 70, 200, 512, torch.bfloat16, False, 3)
    dy = torch.randn(70, 200, device="cuda").to(torch.bfloat16)
    dx, db = hif4.hif4_linear_act_backward(dy, None, w[0], want_dbias=True)             # plain linear: X takes no part
    dx2, none = hif4.hif4_linear_act_backward(dy, x, w[0])
    assert none is None and torch.equal(dx, dx2)
    none, db2 = hif4.hif4_linear_act_backward(dy, x, w[0], want_dx=False, want_dbias=True)
    assert none is None and torch.equal(db, db2)
    wd = decode(hif4, w[0])
    close(dx, dy.double() @ wd, (TOL + 2.0 ** -24) * (dy.double().abs() @ wd.abs()), torch.bfloat16, "dx")
    close(db, dy.double().sum(0), 2.0 ** -17 * dy.double().abs().sum(0), torch.float32, "db")


def test_refusals(hif4):
    x, w, b = operands(hif4, 4, 100, 256, torch.bfloat16, True, 3)
    before = hif4.launch_count()

    def code(f):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        return e.value.code

    assert code(lambda: hif4.hif4_linear_act(x, w[0], act=7)) == 4
    assert code(lambda: hif4.hif4_linear_act(x, w[0], mode=2)) == 4
    assert code(lambda: hif4.hif4_linear_act(x, w[0], units=True)) == 2                        # N % 64
    assert code(lambda: hif4.hif4_linear_act(x, w[0], workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))) == 5
    small = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    assert code(lambda: hif4.hif4_linear_act(x, w[0], workspace=small[1:])) == 3
    odd = torch.zeros(4, 300, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: hif4.hif4_linear_act(odd[:, 1:257], w[0])) == 3                       # rows of X off 16 bytes
    assert code(lambda: hif4.hif4_linear_act(x, w[0], out=torch.zeros(1, 100, dtype=torch.bfloat16, device="cuda").expand(4, 100))) == 2
    dy32 = torch.zeros(4, 100, device="cuda")
    assert code(lambda: hif4.hif4_linear_act_backward(dy32, x.float(), w[0])) == 4            # FP32 gradients
    dy = dy32.to(torch.bfloat16)
    assert code(lambda: hif4.hif4_linear_act_backward(dy, None, w[0], act=2)) == 1
    assert code(lambda: hif4.hif4_gated_linear_backward(dy, None, w[0], w[1])) == 1
    for bad in (lambda: hif4.hif4_linear_act(x, w[0], b[0][:50]), lambda: hif4.hif4_linear_act(x, w[0], b[0].float()),
                lambda: hif4.hif4_linear_act(x, w[0], residual=x), lambda: hif4.hif4_gated_linear(x, w[0], w[1][:50]),
                lambda: hif4.hif4_linear_act(x[:, :192], w[0]), lambda: hif4.hif4_linear_act(x.cpu(), w[0]),
                lambda: hif4.hif4_linear_act(x.t(), w[0]), lambda: hif4.hif4_linear_act_backward(dy, x[:2], w[0], act=2)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        hif4.hif4_linear_act(x.double(), w[0])
    assert hif4.launch_count() == before
