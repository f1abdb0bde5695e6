"""hif4_block_norm and its gradient against the formulas in 64 bits.

Tolerances.  A result is rounded once to its type (relative u: 2^-8 BF16, 2^-11 FP16, 2^-24 FP32); before that it carries
FP32 rounding errors: an element passes fewer than 16 roundings and each row sum, taken as a tree over at most 32 serial
terms per thread and two 5-step butterflies, fewer than 64, so 2^-18 (64 * 2^-24) of the magnitudes that enter it bounds
the arithmetic."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}
ARITH = 2.0 ** -18
EPS = 1e-5


@pytest.fixture(scope="module")
def hif4():
    assert torch.cuda.is_available()
    import paper_2602_11287_b200 as lib
    return lib


def _std(v, kind):
    if kind == 0:
        return v
    if kind == 2:
        v = v - v.mean(1, keepdim=True)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)


def forward64(x, r, scale, gate, rpg, post, wp, pre, w, b):
    p = _std(x, post)
    if wp is not None:
        p = p * wp
    g = 1.0 if gate is None else gate[torch.arange(x.shape[0], device=x.device) // rpg]
    h = g * p + (scale * r if r is not None else 0.0)
    if pre == 0:
        return h, None
    y = _std(h, pre)
    y = y * w if w is not None else y
    return h, y + b if b is not None else y


def close(got, ref, mag, dtype, what):
    """|got - ref| <= u |ref| + ARITH * mag (+ half the smallest step of the type)."""
    err = (got.double() - ref).abs()
    bound = U[dtype] * ref.abs() + ARITH * mag + TINY[dtype]
    worst = float((err / bound).max()) if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: worst ratio {worst:.3g}"


def make(rows, cols, dtype, wtype, post, pre, rpg, res, seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    x = (rnd(rows, cols) * 2).to(dtype)
    r = (rnd(rows, cols) * 3).to(dtype) if res else None
    gate = (1 + 0.5 * rnd(-(-rows // rpg), cols)).to(dtype) if rpg else None
    wp = (1 + 0.3 * rnd(cols)).to(wtype) if post else None
    w = (1 + 0.3 * rnd(cols)).to(wtype)
    b = rnd(cols).to(wtype) if pre == 2 else None
    return x, r, gate, wp, w, b


def d64(*ts):
    return [None if t is None else t.double() for t in ts]


def check_forward(hif4, x, r, gate, wp, w, b, scale, rpg, post, pre, what, **kw):
    dtype = x.dtype
    h, y = hif4.hif4_block_norm(x, w, b, residual=r, res_scale=scale, gate=gate, rows_per_gate=rpg, post=post, post_weight=wp,
                                pre=pre, eps=EPS, **kw)
    X, R, G, WP, W, B = d64(x, r, gate, wp, w, b)
    H, Y = forward64(X, R, scale, G, rpg, post, WP, pre, W, B)
    magh = H.abs() + (scale * R).abs() if r is not None else H.abs()
    rows_mag = magh.amax(1, keepdim=True)
    close(h, H, magh + (X.abs().amax(1, keepdim=True) if post else 0.0), dtype, what + " h")
    rstd = 1.0 / torch.sqrt((_std_centre(H, pre) ** 2).mean(1, keepdim=True) + EPS)
    magy = rows_mag * rstd * W.abs() + (B.abs() if b is not None else 0.0)
    close(y, Y, magy, dtype, what + " y")
    return h, y


def _std_centre(v, kind):
    return v - v.mean(1, keepdim=True) if kind == 2 else v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 8), (2, 64), (7, 100), (5, 1001), (33, 256), (300, 1000),
                                       (9, 4104), (4, 8192), (3, 8200), (2, 16384), (2, 20000), (1, 32768), (700, 128)])
def test_forward_sizes(hif4, dtype, rows, cols):
    for n, (post, pre, rpg) in enumerate([(0, 1, 0), (1, 2, 1), (2, 1, 3)]):
        t = make(rows, cols, dtype, dtype, post, pre, rpg, n != 0 or rows > 3, 7 * rows + cols + n)
        check_forward(hif4, *t, 0.5, rpg, post, pre, f"{rows}x{cols} post={post} pre={pre} rpg={rpg}")


@pytest.mark.parametrize("dtype,wtype", itertools.product([torch.bfloat16, torch.float16, torch.float32], repeat=2))
def test_weight_types_and_strides(hif4, dtype, wtype):
    rows, cols = 37, 264
    x, r, gate, wp, w, b = make(rows, cols, dtype, wtype, 1, 2, 5, True, 3)
    big = torch.zeros(rows, 3, 280, dtype=dtype, device="cuda")
    # row strides that keep 16-byte accesses, an odd base, and odd strides
    for off, view in ((8, big[:, 1]), (1, big[:, 1]), (3, torch.zeros(rows, 271, dtype=dtype, device="cuda"))):
        xs = view[:, off:off + cols]
        xs.copy_(x)
        guard = torch.full((rows + 2, cols + 24), 7.0, dtype=dtype, device="cuda")
        gy = guard.clone()
        check_forward(hif4, xs, r, gate, wp, w, b, 0.7, 5, 1, 2, f"off {off}", out_h=guard[1:-1, 8:8 + cols], out_y=gy[1:-1, 16:16 + cols])
        for t, o in ((guard, 8), (gy, 16)):
            t[1:-1, o:o + cols] = 7.0
            assert (t == 7.0).all(), "written outside the matrix"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("rows,cols,off", [(1, 64, 0), (5, 192, 0), (40, 4096, 0), (3, 5120, 0), (2, 16384, 0), (6, 320, 1)])
def test_units_are_the_quantized_rows(hif4, dtype, mode, rows, cols, off):
    x, r, gate, wp, w, b = make(rows, cols + off, dtype, dtype, 1, 1, 0, True, cols)
    kw = dict(residual=r[:, off:], res_scale=0.9, post=1, post_weight=wp[off:], eps=EPS)
    h, y = hif4.hif4_block_norm(x[:, off:], w[off:], **kw)
    h2, u = hif4.hif4_block_norm(x[:, off:], w[off:], units=True, mode=mode, **kw)
    assert torch.equal(h, h2) and torch.equal(u, hif4.hif4_quantize(y, mode=mode))


def test_units_of_unusual_rows(hif4):
    """Zeros, a single spike, infinities and NaN: the row statistics follow the formula, the units are those of y."""
    x = torch.zeros(6, 256, dtype=torch.bfloat16, device="cuda")
    x[1, 5], x[2, 7], x[3, 100] = 3.0, float("inf"), float("nan")
    x[4] = -0.0
    x[5] = 1e30
    for dtype in (torch.bfloat16, torch.float32):
        h, y = hif4.hif4_block_norm(x.to(dtype), None)
        _, u = hif4.hif4_block_norm(x.to(dtype), None, units=True)
        assert torch.equal(u, hif4.hif4_quantize(y))
        assert torch.equal(y[0], torch.zeros_like(y[0])) and torch.isnan(y[3]).all() and torch.isnan(y[2, 7])
        assert torch.equal(y[2, :7], torch.zeros_like(y[2, :7]))
    assert hif4.hif4_last_device_status() == 0


def test_h_in_place_nothing_to_do_and_empty(hif4):
    x, r, gate, wp, w, b = make(50, 512, torch.bfloat16, torch.bfloat16, 0, 1, 0, True, 5)
    h, y = hif4.hif4_block_norm(x, w, residual=r)
    for target in ("x", "r"):
        x2, r2 = x.clone(), r.clone()
        h2, y2 = hif4.hif4_block_norm(x2, w, residual=r2, out_h=x2 if target == "x" else r2)
        assert torch.equal(h, h2) and torch.equal(y, y2)
    h3, y3 = hif4.hif4_block_norm(x, w)
    assert h3 is x
    h4, y4 = hif4.hif4_block_norm(x, None, residual=r, pre=hif4.HIF4_NORM_NONE)
    assert y4 is None and torch.equal(h4, h)
    h5, y5 = hif4.hif4_block_norm(x[:0], w, residual=r[:0])
    assert y5.shape == (0, 512)
    d = hif4.hif4_block_norm_backward(y5, h5, w, bias=True, pre=hif4.HIF4_NORM_LAYER)
    assert (d["dweight"] == 0).all() and (d["dbias"] == 0).all()


def test_other_stream(hif4):
    x, r, gate, wp, w, b = make(2000, 2048, torch.bfloat16, torch.bfloat16, 1, 1, 0, True, 9)
    want = hif4.hif4_block_norm(x, w, residual=r, post=1, post_weight=wp)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(20):
        outs.append(hif4.hif4_block_norm_backward(x, r, w, dh=x, x=r, post=1, post_weight=wp, stream=s))
        torch.empty(5 * 296 * 2048 * 4, dtype=torch.uint8, device="cuda").fill_(255)      # would land in a workspace given back too early
    got = hif4.hif4_block_norm(x, w, residual=r, post=1, post_weight=wp, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for o in outs[1:]:
        assert all(torch.equal(o[k], outs[0][k]) for k in o if o[k] is not None)


# ------------------------------------------------------------------------------------------------------------ gradients
def reference_grads(x, r, gate, wp, w, b, scale, rpg, post, pre, h, dy, dh):
    """Autograd of the formulas in 64 bits.  The norm is differentiated at the stored h, as the call does."""
    X, R, G, WP, W, B, DY, DH = d64(x, r, gate, wp, w, b, dy, dh)
    H = h.double().requires_grad_()
    leaves = [t.requires_grad_() for t in (W, B) if t is not None]
    y = _std(H, pre) * W
    y = y + B if b is not None else y
    gh, *gw = torch.autograd.grad(y, [H, *leaves], DY)
    total = gh + DH
    leaves2 = [t.requires_grad_() for t in (X, R, G, WP) if t is not None]
    h2, _ = forward64(X, R, scale, G, rpg, post, WP, 0, None, None)
    g2 = list(torch.autograd.grad(h2, leaves2, total))
    out = {"dweight": gw[0], "dbias": gw[1] if b is not None else None}
    for k, t in (("dx", X), ("dresidual", R), ("dgate", G), ("dpost_weight", WP)):
        out[k] = g2.pop(0) if t is not None else None
    return out, total


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (2, 100), (17, 64), (200, 1001), (1000, 512), (300, 4096), (65, 8192), (7, 16384), (3, 17000)])
@pytest.mark.parametrize("post,pre,rpg", [(0, 1, 0), (1, 1, 0), (2, 2, 1), (0, 2, 7), (1, 2, 600)])
def test_gradients(hif4, dtype, rows, cols, post, pre, rpg):
    x, r, gate, wp, w, b = make(rows, cols, dtype, dtype, post, pre, rpg, True, rows + 3 * cols + post)
    g = torch.Generator(device="cuda"); g.manual_seed(11)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    dh = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    scale = 0.5
    h, _ = hif4.hif4_block_norm(x, w, b, residual=r, res_scale=scale, gate=gate, rows_per_gate=rpg, post=post, post_weight=wp, pre=pre, eps=EPS)
    d = hif4.hif4_block_norm_backward(dy, h, w, dh=dh, x=x, bias=b is not None, res_scale=scale, gate=gate, rows_per_gate=rpg,
                                      post=post, post_weight=wp, pre=pre, eps=EPS)
    want, total = reference_grads(x, r, gate, wp, w, b, scale, rpg, post, pre, h, dy, dh)
    X, R, G, WP, W, B = d64(x, r, gate, wp, w, b)
    H = h.double()
    rstd = 1.0 / torch.sqrt((_std_centre(H, pre) ** 2).mean(1, keepdim=True) + EPS)
    # magnitudes: every term of the row formulas is at most max |dn| (1 + |n|max^2) rstd
    n = _std(H, pre).abs()
    if pre == 2:          # the centred value carries the rounding of h - mean
        n = n + H.abs().amax(1, keepdim=True) * rstd
    dn = (dy.double() * W).abs().amax(1, keepdim=True)
    magt = dh.double().abs() + rstd * dn * (1 + n * n.amax(1, keepdim=True))
    close(d["dresidual"], want["dresidual"], scale * magt, dtype, "dresidual")
    gg = torch.ones_like(X) if gate is None else G[torch.arange(rows, device="cuda") // rpg].abs()
    if post:
        rx = 1.0 / torch.sqrt((_std_centre(X, post) ** 2).mean(1, keepdim=True) + EPS)
        nx = _std(X, post).abs() + (X.abs().amax(1, keepdim=True) * rx if post == 2 else 0.0)
        dq = (magt * gg * WP.abs()).amax(1, keepdim=True)
        magx = rx * dq * (1 + nx * nx.amax(1, keepdim=True))
        p = nx * WP.abs()
    else:
        nx, p, magx = X.abs(), X.abs(), magt * gg
    close(d["dx"], want["dx"], magx, dtype, "dx")
    # column sums: serial over a block's rows, then over the blocks
    serial = 2.0 ** -24 * (64 + rows / 148 + 300) / ARITH
    f32 = torch.float32
    close(d["dweight"], want["dweight"], serial * (dy.double().abs() * n).sum(0), f32, "dweight")
    if b is not None:
        close(d["dbias"], want["dbias"], serial * dy.double().abs().sum(0), f32, "dbias")
    if post:
        close(d["dpost_weight"], want["dpost_weight"], serial * (magt * gg * nx).sum(0), f32, "dpost_weight")
    if gate is not None:
        mag = torch.zeros_like(G).index_add_(0, torch.arange(rows, device="cuda") // rpg, magt * p)
        close(d["dgate"], want["dgate"], serial * mag, dtype, "dgate")


def test_gradient_against_differences(hif4):
    """FP32: the gradient's product with a direction against the centred difference of <y, cy> + <h, ch>.  The difference
    of step e carries e^2 times third derivatives (order one here) and 2^-24 / e of rounding: 1e-4 at e = 3e-3."""
    rows, cols, scale, rpg = 12, 96, 0.6, 5
    x, r, gate, wp, w, b = make(rows, cols, torch.float32, torch.float32, 1, 2, rpg, True, 21)
    g = torch.Generator(device="cuda"); g.manual_seed(4)
    cy, ch = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(2))

    def f(x, r, gate, wp, w, b):
        h, y = hif4.hif4_block_norm(x, w, b, residual=r, res_scale=scale, gate=gate, rows_per_gate=rpg, post=1, post_weight=wp, pre=2, eps=EPS)
        return (y.double() * cy.double()).sum() + (h.double() * ch.double()).sum()

    h, _ = hif4.hif4_block_norm(x, w, b, residual=r, res_scale=scale, gate=gate, rows_per_gate=rpg, post=1, post_weight=wp, pre=2, eps=EPS)
    d = hif4.hif4_block_norm_backward(cy, h, w, dh=ch, x=x, bias=True, res_scale=scale, gate=gate, rows_per_gate=rpg, post=1, post_weight=wp, pre=2, eps=EPS)
    args = [x, r, gate, wp, w, b]
    for i, k in enumerate(("dx", "dresidual", "dgate", "dpost_weight", "dweight", "dbias")):
        v = torch.randn(args[i].shape, generator=g, device="cuda")
        e = 3e-3
        up, down = ([a + s * e * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        diff = float((f(*up) - f(*down)) / (2 * e))
        got = float((d[k].double() * v.double()).sum())
        size = float((d[k].double().abs() * v.double().abs()).sum())
        assert abs(diff - got) <= 1e-3 * size, (k, diff, got)


def test_gradients_that_are_not_wanted(hif4):
    rows, cols = 90, 320
    x, r, gate, wp, w, b = make(rows, cols, torch.bfloat16, torch.float32, 0, 1, 0, True, 2)
    full = hif4.hif4_block_norm_backward(x, r, w, dh=x)
    part = hif4.hif4_block_norm_backward(x, r, w, dh=x, want_dresidual=False)
    assert part["dresidual"] is None and torch.equal(part["dx"], full["dx"]) and torch.equal(part["dweight"], full["dweight"])
    zero = torch.zeros_like(x)
    a = hif4.hif4_block_norm_backward(x, r, w)                                # no gradient from the residual stream
    assert torch.equal(a["dx"], hif4.hif4_block_norm_backward(x, r, w, dh=zero)["dx"])
    c = hif4.hif4_block_norm_backward(None, None, None, dh=x, res_scale=0.5)  # no norm in front
    assert torch.equal(c["dx"], x) and torch.equal(c["dresidual"], (x.float() * 0.5).to(x.dtype)) and c["dweight"] is None


def test_refusals(hif4):
    x = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(128, dtype=torch.bfloat16, device="cuda")
    before = hif4.launch_count()

    def code(f):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        return e.value.code

    assert code(lambda: hif4.hif4_block_norm(x, w, bias=w)) == 2                                     # bias of an RMS norm
    assert code(lambda: hif4.hif4_block_norm(x, w, eps=-1.0)) == 2
    assert code(lambda: hif4.hif4_block_norm(x, w, eps=float("nan"))) == 2
    assert code(lambda: hif4.hif4_block_norm(x, w, pre=5)) == 4
    assert code(lambda: hif4.hif4_block_norm(x, w, mode=3, units=True)) == 4
    assert code(lambda: hif4.hif4_block_norm(x[:, :100], w[:100], units=True)) == 2
    assert code(lambda: hif4.hif4_block_norm(torch.zeros(1, 32776, dtype=torch.bfloat16, device="cuda"))) == 2
    assert code(lambda: hif4.hif4_block_norm(x, w, pre=0, out_y=x.clone())) == 2
    assert code(lambda: hif4.hif4_block_norm(x[:1].expand(4, 128), w)) == 2                           # rows over one another
    assert code(lambda: hif4.hif4_block_norm_backward(x, None, w)) == 1
    assert code(lambda: hif4.hif4_block_norm_backward(x, x, w, post=1, post_weight=w)) == 1           # x is missing
    assert code(lambda: hif4.hif4_block_norm_backward(x, x, w, post_weight=w)) == 2                   # weight of no norm
    assert code(lambda: hif4.hif4_block_norm_backward(x, x, w, bias=True)) == 2                       # bias of an RMS norm
    assert code(lambda: hif4.hif4_block_norm_backward(x, x, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))) == 5
    for bad in (lambda: hif4.hif4_block_norm(x, w[:100]), lambda: hif4.hif4_block_norm(x, w, residual=x[:2]),
                lambda: hif4.hif4_block_norm(x, w, residual=x.float()), lambda: hif4.hif4_block_norm(x, w, gate=x[:1]),
                lambda: hif4.hif4_block_norm(x.cpu(), w.cpu()), lambda: hif4.hif4_block_norm(x.t(), None),
                lambda: hif4.hif4_block_norm(x[0], w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        hif4.hif4_block_norm(x.double(), None)
    assert hif4.launch_count() == before
