"""MXFP4 and NVFP4: conversion, its inverse, products and grouped products against the definitions."""
import pytest
import torch

from tests import bfp4_reference as ref

pytestmark = pytest.mark.gpu
MX, NV = 1, 2


@pytest.fixture(scope="module")
def hif4():
    import paper_2602_11287_b200 as m
    return m


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def matrix(rows, cols, dtype, seed):
    """Rows of many magnitudes, with zeros, negative zeros, a block of zeros and exact ties."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 10, (rows, 1), generator=g, device="cuda").float())
    x[:, ::7] = 0.0
    x[:, 1::11] = -0.0
    x[rows // 2, : min(64, cols)] = 0.0
    tie = torch.tensor([6.0, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5.0], device="cuda")
    x[0, :64] = tie.repeat(8)
    return x.to(dtype)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols,gain", [(1, 64, None), (3, 192, 1.7), (130, 1024, None), (77, 4160, 0.01), (1024, 320, None)])
def test_conversion(hif4, fmt, dtype, rows, cols, gain):
    x = matrix(rows, cols, dtype, rows + cols)
    g = None if gain is None else torch.full((1,), gain, device="cuda")
    codes, scales = hif4.hif4_bfp4_quantize(x, fmt, gain=g)
    want = ref.pack(*ref.convert(x, fmt, g))
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    v = ref.values(*want, fmt)
    for dt in (torch.bfloat16, torch.float32):
        got = hif4.hif4_bfp4_dequantize((codes, scales), fmt, dt, gain=g)
        assert torch.equal(got, v.to(dt) if g is None else (v.float() / g).to(dt))


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gain", [-0.7, 1e-30, 1e30, 3e38, 2.0 ** -140, 0.0, float("nan")])
def test_gains_of_any_size(hif4, fmt, dtype, gain):
    x = matrix(20, 320, dtype, 11)
    g = torch.full((1,), gain, device="cuda")
    codes, scales = hif4.hif4_bfp4_quantize(x, fmt, gain=g)
    want = ref.pack(*ref.convert(x, fmt, g))
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    for dt in (torch.bfloat16, torch.float32):
        got, v = hif4.hif4_bfp4_dequantize((codes, scales), fmt, dt, gain=g), (ref.values(*want, fmt).float() / g).to(dt)
        assert torch.equal(got.isnan(), v.isnan()) and torch.equal(got.nan_to_num(0.0, 1e38, -1e38), v.nan_to_num(0.0, 1e38, -1e38))
        assert torch.equal(torch.signbit(got[~got.isnan()]), torch.signbit(v[~v.isnan()]))


@pytest.mark.parametrize("fmt", [MX, NV])
def test_image_is_the_quantization_study_s(hif4, fmt):
    x = matrix(64, 1024, torch.bfloat16, 5)
    image, _ = hif4.hif4_mse_roundtrip(x, fmt)
    assert torch.equal(hif4.hif4_bfp4_dequantize(hif4.hif4_bfp4_quantize(x, fmt), fmt, torch.float32), image)


@pytest.mark.parametrize("fmt", [MX, NV])
def test_every_bf16_quotient(hif4, fmt):
    """Each block: one peak and fifteen (thirty-one) numbers of every size below it."""
    n = BL = ref.BLOCK[fmt]
    peak = torch.arange(0x3F80, 0x4100, device="cuda", dtype=torch.int32)                     # 1 <= peak < 8
    frac = torch.arange(1, 256 * (n - 1) + 1, device="cuda").float() / (256 * (n - 1))
    x = (peak.to(torch.int16).view(torch.bfloat16).float().view(-1, 1, 1) * frac.view(1, 256, n - 1)).to(torch.bfloat16)
    top = peak.to(torch.int16).view(torch.bfloat16).view(-1, 1, 1).expand(-1, 256, 1)
    x = torch.cat([top, x], 2).reshape(-1, 64 * BL // BL)
    codes, scales = hif4.hif4_bfp4_quantize(x, fmt)
    want = ref.pack(*ref.convert(x, fmt))
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_values(hif4, fmt, dtype):
    x = matrix(8, 256, dtype, 3).float()
    x[0, 5], x[1, 40], x[2, 70], x[2, 71] = torch.nan, torch.inf, -torch.inf, 1.0
    x[3] *= 1e38 / x[3].abs().max()
    x[4] = torch.where(x[4] == 0, x[4], torch.sign(x[4]) * 1e-38)
    x[5, :32] = 1e-40
    x = x.to(dtype)
    codes, scales = hif4.hif4_bfp4_quantize(x, fmt)
    want = ref.pack(*ref.convert(x, fmt))
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    back = hif4.hif4_bfp4_dequantize((codes, scales), fmt, torch.float32)
    v = ref.values(*want, fmt).float()
    assert torch.equal(back.isnan(), v.isnan()) and torch.equal(back.nan_to_num(0.0), v.nan_to_num(0.0))


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(64, 8), (64, 136), (320, 1000), (1024, 40), (256, 72), (768, 264), (1088, 128)])
def test_conversion_down_the_columns(hif4, fmt, dtype, rows, cols):
    x = matrix(rows, max(cols, 64), dtype, rows + cols)[:, :cols]
    g = torch.full((1,), 0.3, device="cuda") if cols == 136 else None
    got = hif4.hif4_bfp4_quantize_transposed(x, fmt, gain=g)
    want = hif4.hif4_bfp4_quantize(x.t().contiguous(), fmt, gain=g)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_conversion_of_a_view_leaves_its_surroundings(hif4):
    x = matrix(9, 256, torch.bfloat16, 1)
    wide = torch.full((9, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 128:384] = x
    a, b = hif4.hif4_bfp4_quantize(wide[:, 128:384], NV), hif4.hif4_bfp4_quantize(x, NV)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out = torch.full((9, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    hif4.hif4_bfp4_dequantize(a, NV, out=out[:, 128:384])
    assert torch.equal(out[:, 128:384], hif4.hif4_bfp4_dequantize(b, NV))
    assert bool((out[:, :128] == 7).all() and (out[:, 384:] == 7).all())


def check_product(y, a, b, scale=1.0):
    """FP32 sums in any order: the bound of the HiF4 product; then one rounding to the type of Y."""
    want, most = scale * (a @ b.t()), abs(scale) * 1e-5 * (a.abs() @ b.abs().t())
    most = most + torch.finfo(y.dtype).eps / 2 * want.abs() * (0 if y.dtype == torch.float32 else 1) + 2.0 ** -24 * want.abs()
    if y.dtype == torch.float16:          # below 2^-14 FP16's step is 2^-24 whatever the value: half of it is 2^-25
        most = most + 2.0 ** -25
    assert bool(((y.double() - want).abs() <= most).all()), float(((y.double() - want).abs() / most.clamp(min=1e-300)).max())


SIZES = [(1, 1, 64), (1, 8, 128), (1, 300, 256), (2, 129, 320), (7, 128, 512), (16, 256, 576), (17, 513, 1024), (33, 64, 2048),
         (64, 1000, 4096), (65, 130, 192), (128, 384, 1088), (129, 257, 768), (300, 200, 8256), (513, 777, 320), (1024, 512, 1024),
         (200, 1, 1024), (70, 9, 2048), (66, 40, 4096)]


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(hif4, fmt, M, N, K):
    g = gen(M + N + K)
    a, b = ref.random_operand(M, K, fmt, g), ref.random_operand(N, K, fmt, g)
    A, B = ref.values(*a, fmt), ref.values(*b, fmt)
    alpha = torch.full((1,), 0.37, device="cuda")
    check_product(hif4.hif4_bfp4_gemm(a, b, fmt, dtype=torch.float32), A, B)
    check_product(hif4.hif4_bfp4_gemm(a, b, fmt, alpha=alpha), A, B, float(alpha))
    check_product(hif4.hif4_bfp4_gemm(a, b, fmt, alpha=alpha / 64, dtype=torch.float16), A, B, float(alpha / 64))
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,K", [(1500, 1777, 320), (2049, 2304, 1088), (257, 9600, 576), (8200, 512, 64), (1300, 2050, 2304), (2560, 2560, 512),
                                   (700, 2836, 1024), (333, 1001, 320), (70, 131, 832)])
def test_product_of_prompts(hif4, fmt, M, N, K):
    """The sizes of the CTA-pair kernel."""
    test_product(hif4, fmt, M, N, K)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M", [1, 40, 200, 10000])
def test_every_code_and_scale(hif4, fmt, M):
    """One row of A picks one element of each row of B: products are exact."""
    K = 512
    bytes_ = torch.arange(0, 255 if fmt == MX else 127, device="cuda")
    usable = bytes_[(bytes_ > 20) & (bytes_ < 235)] if fmt == MX else bytes_
    N = usable.numel()
    code = torch.arange(K, device="cuda").remainder(16).expand(N, K).to(torch.uint8)
    b = ref.pack(code, usable.view(N, 1).expand(N, K // ref.BLOCK[fmt]).to(torch.uint8))
    pick = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16)
    pick[torch.arange(M), (torch.arange(M) * 37) % K] = 6.0
    a = hif4.hif4_bfp4_quantize(pick, fmt)
    want = pick.double() @ ref.values(*b, fmt).t()
    assert torch.equal(hif4.hif4_bfp4_gemm(a, b, fmt, dtype=torch.float32).double(), want)


@pytest.mark.parametrize("fmt", [MX, NV])
def test_nan_blocks_and_row_padding(hif4, fmt):
    """A NaN scale makes the outputs of its row NaN; scale bytes past the last block are never read."""
    g = gen(1)
    a, b = ref.random_operand(20, 320, fmt, g), ref.random_operand(150, 320, fmt, g)
    clean = hif4.hif4_bfp4_gemm(a, b, fmt, dtype=torch.float32)
    used = 320 // ref.BLOCK[fmt]
    for q in (a, b):
        q[1][used // 16, :, used % 16:] = 255 if fmt == MX else 127
    assert torch.equal(hif4.hif4_bfp4_gemm(a, b, fmt, dtype=torch.float32), clean)
    a[1][0, 3, 2] = b[1][0, 140, 1] = 255 if fmt == MX else 127
    got = hif4.hif4_bfp4_gemm(a, b, fmt, dtype=torch.float32)
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[3], nan[:, 140] = True, True
    assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan], clean[~nan])


@pytest.mark.parametrize("M", [5, 100, 300, 10000])
def test_product_into_a_view(hif4, M):
    g = gen(2)
    a, b = ref.random_operand(M, 1024, NV, g), ref.random_operand(203, 1024, NV, g)
    for dt in (torch.bfloat16, torch.float32):
        wide = torch.full((M + 2, 301), 3.0, dtype=dt, device="cuda")
        hif4.hif4_bfp4_gemm(a, b, NV, out=wide[1:M + 1, 50:253])
        assert torch.equal(wide[1:M + 1, 50:253], hif4.hif4_bfp4_gemm(a, b, NV, dtype=dt))
        wide[1:M + 1, 50:253] = 3.0
        assert bool((wide == 3.0).all())


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("counts,N,K", [([3], 100, 64), ([0, 1, 0, 0, 17, 0], 130, 320), ([40, 0, 129, 1, 300], 257, 512), ([5] * 40, 128, 1024),
                                        ([0, 0], 64, 128), ([600, 1, 1], 320, 2112),
                                        ([20, 0, 70, 33, 64, 1], 520, 4096), ([700, 0, 333, 1], 520, 320), ([256, 512, 17], 300, 1088), ([1000, 31], 257, 128), ([500, 140, 0, 141], 1002, 192), ([1, 2, 0] * 100, 64, 320), ([7] * 256, 130, 576)])
def test_grouped_product(hif4, fmt, counts, N, K):
    g = gen(sum(counts) + N)
    G, used = len(counts), sum(counts)
    R = used + 19                                                # rows behind the last group
    a, b = ref.random_operand(R, K, fmt, g), ref.random_operand(N, K, fmt, g, groups=G)
    off = torch.tensor([0] + counts, device="cuda").cumsum(0)
    alpha = torch.rand(G, generator=g, device="cuda") + 0.5
    A, B = ref.values(*a, fmt), ref.values(*b, fmt)
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((R, N), 9.0, dtype=dt, device="cuda")
        assert hif4.hif4_bfp4_grouped_gemm(a, b, off, fmt, alpha=alpha, out=y) is y
        for n in range(G):
            check_product(y[off[n]:off[n + 1]], A[off[n]:off[n + 1]], B[n], float(alpha[n]))
        assert bool((y[used:] == 9.0).all())
    assert hif4.hif4_last_device_status() == 0


def test_offsets_outside_the_rows_are_clamped(hif4):
    g = gen(4)
    a, b = ref.random_operand(50, 256, NV, g), ref.random_operand(64, 256, NV, g, groups=3)
    good = torch.tensor([0, 20, 20, 50], device="cuda")
    want = hif4.hif4_bfp4_grouped_gemm(a, b, good, NV)
    assert torch.equal(hif4.hif4_bfp4_grouped_gemm(a, b, torch.tensor([-7, 20, 20, 50], device="cuda"), NV), want)
    pool = torch.full((60, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    hif4.hif4_bfp4_grouped_gemm(a, b, torch.tensor([-7, 60, 5, 2 ** 40], device="cuda"), NV, out=pool[:50])        # not offsets at all
    assert bool((pool[50:] == 2.0).all())
    assert torch.equal(hif4.hif4_bfp4_grouped_gemm(a, b, torch.tensor([0, 20, 20, 2 ** 40], device="cuda"), NV), want)


def test_gradients_of_a_linear_layer(hif4):
    """dX and dW from operands converted down the columns, against the formulas on the converted operands."""
    g = gen(6)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    M, N, K = 192, 320, 256
    x, w, dy = rnd(M, K), rnd(N, K) / 16, rnd(M, N)
    for fmt in (MX, NV):
        V = lambda q: ref.values(*q, fmt)      # noqa: E731
        qd, wt = hif4.hif4_bfp4_quantize(dy, fmt), hif4.hif4_bfp4_quantize_transposed(w, fmt)
        check_product(hif4.hif4_bfp4_gemm(qd, wt, fmt, dtype=torch.float32), V(qd), V(wt))
        dt, xt = hif4.hif4_bfp4_quantize_transposed(dy, fmt), hif4.hif4_bfp4_quantize_transposed(x, fmt)
        dw = hif4.hif4_bfp4_gemm(dt, xt, fmt, dtype=torch.float32)
        check_product(dw, V(dt), V(xt))
        # a 4-bit element is off by at most a quarter of its block's peak; in the mean far less
        assert float((dw.double() - dy.double().t() @ x.double()).norm() / (dy.double().t() @ x.double()).norm()) < 0.25


def test_same_bits_every_time_and_in_a_graph(hif4):
    g = gen(8)
    for M in (1, 30, 100, 700, 3500):
        a, b = ref.random_operand(M, 4096, NV, g), ref.random_operand(520, 4096, NV, g)
        y = hif4.hif4_bfp4_gemm(a, b, NV, dtype=torch.float32)
        out = torch.empty_like(y)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            hif4.hif4_bfp4_gemm(a, b, NV, out=out)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                hif4.hif4_bfp4_gemm(a, b, NV, out=out)
        torch.cuda.current_stream().wait_stream(s)
        for _ in range(3):
            out.zero_()
            graph.replay()
            assert torch.equal(out, y)


def test_refusals(hif4):
    x = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")
    q = hif4.hif4_bfp4_quantize(x, NV)
    w = q[0].view(1, 64, 128), q[1].view(1, 1, 64, 16)
    off = torch.tensor([0, 64], device="cuda")
    for f in (lambda: hif4.hif4_bfp4_quantize(x, 0), lambda: hif4.hif4_bfp4_quantize(x, 3), lambda: hif4.hif4_bfp4_quantize(x, 2 ** 32 + 1),
              lambda: hif4.hif4_bfp4_dequantize(q, NV, torch.float16), lambda: hif4.hif4_bfp4_gemm(q, q, 0)):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        assert e.value.code == 4
    for f in (lambda: hif4.hif4_bfp4_quantize(x[:, :100], NV), lambda: hif4.hif4_bfp4_quantize_transposed(x[:50], NV),
              lambda: hif4.hif4_bfp4_quantize_transposed(x[:, :100], NV)):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        assert e.value.code == 2
    with pytest.raises(hif4.Hif4Error) as e:
        hif4.hif4_bfp4_quantize(x.view(-1)[1:1 + 63 * 256].view(63, 256), NV)
    assert e.value.code == 3
    for f in (lambda: hif4.hif4_bfp4_quantize(x, NV, gain=torch.ones(2, device="cuda")), lambda: hif4.hif4_bfp4_quantize(x.t(), NV),
              lambda: hif4.hif4_bfp4_dequantize((q[0], q[1][:, :32]), NV), lambda: hif4.hif4_bfp4_gemm(q, (q[0][:, :64].contiguous(), q[1]), NV),
              lambda: hif4.hif4_bfp4_gemm(q, q, NV, alpha=torch.ones(1, dtype=torch.float64, device="cuda")),
              lambda: hif4.hif4_bfp4_grouped_gemm(q, q, off, NV), lambda: hif4.hif4_bfp4_grouped_gemm(q, w, off.int(), NV),
              lambda: hif4.hif4_bfp4_grouped_gemm(q, w, off, NV, alpha=torch.ones(2, device="cuda")),
              lambda: hif4.hif4_bfp4_gemm(q, q, NV, out=torch.empty(64, 63, device="cuda")), lambda: hif4.hif4_bfp4_quantize(x.cpu(), NV)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: hif4.hif4_bfp4_gemm(q[0], q, NV), lambda: hif4.hif4_bfp4_gemm(q, (q[0],), NV), lambda: hif4.hif4_bfp4_quantize(x.double(), NV),
              lambda: hif4.hif4_bfp4_grouped_gemm(q, w, None, NV)):
        with pytest.raises(TypeError):
            f()


def test_empty_sizes(hif4):
    e = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    q = hif4.hif4_bfp4_quantize(e, NV)
    full = hif4.hif4_bfp4_quantize(torch.ones(5, 256, dtype=torch.bfloat16, device="cuda"), NV)
    assert q[0].shape == (0, 128) and q[1].shape == (1, 0, 16)
    assert hif4.hif4_bfp4_gemm(q, full, NV).shape == (0, 5) and hif4.hif4_bfp4_gemm(full, q, NV).shape == (5, 0)
    assert hif4.hif4_bfp4_dequantize(q, NV).shape == (0, 256)
