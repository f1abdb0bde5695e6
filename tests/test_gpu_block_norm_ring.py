"""The block norms' ring of shared-memory stages (many long aligned rows) against the formulas in 64 bits: sizes at which every
block takes more rows than the ring has stages, so that stages are filled again.  Tolerances as in test_gpu_block_norm.py."""
import pytest
import torch

from tests.test_gpu_block_norm import ARITH, EPS, TINY, U, check_forward, hif4, make  # noqa: F401
from tests.test_gpu_block_norm import test_gradients as check_gradients

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# rows a block at 148 SMs: 10 (six blocks an SM), 9 (six), 8 (two), 8 (two) or 16 (one), 4 (one)
FORWARD = [(9000, 1024), (8000, 2048), (2500, 5120), (2500, 8192), (700, 20000)]
KINDS = [(0, 1, 0), (1, 2, 1), (2, 1, 3), (1, 1, 700), (0, 2, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", FORWARD)
@pytest.mark.parametrize("post,pre,rpg", KINDS)
def test_forward(hif4, dtype, rows, cols, post, pre, rpg):
    check_forward(hif4, *make(rows, cols, dtype, dtype, post, pre, rpg, True, rows + post + pre), 0.5, rpg, post, pre,
                  f"{rows}x{cols} post={post} pre={pre} rpg={rpg}")
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forward_without_residual(hif4, dtype):
    check_forward(hif4, *make(2500, 4096, dtype, dtype, 1, 1, 0, False, 4), 0.5, 0, 1, 1, "no residual")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("rows,cols", [(9000, 1024), (2500, 5120), (2500, 8192)])
def test_units_are_the_quantized_rows(hif4, dtype, mode, rows, cols):
    x, r, gate, wp, w, b = make(rows, cols, dtype, dtype, 1, 1, 5, True, cols)
    kw = dict(residual=r, res_scale=0.9, gate=gate, rows_per_gate=5, post=1, post_weight=wp, eps=EPS)
    h, y = hif4.hif4_block_norm(x, w, **kw)
    h2, u = hif4.hif4_block_norm(x, w, units=True, mode=mode, **kw)
    assert torch.equal(h, h2) and torch.equal(u, hif4.hif4_quantize(y, mode=mode))


def strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device="cuda")
    v = wide[:, 8:8 + t.shape[1]]
    v.copy_(t)
    return wide, v


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(8000, 2048), (2500, 5120)])
def test_strides_weight_types_h_alone_and_in_place(hif4, dtype, rows, cols):
    """Other strides (each its own) and h over x or the residual: the same bits.  FP32 weights and h alone may be the direct kernel's,
    whose sums run in another order: FP32 weights against the formula, h alone within the tolerances of two results."""
    x, r, gate, wp, w, b = make(rows, cols, dtype, dtype, 1, 2, 3, True, 17)
    kw = dict(res_scale=0.5, rows_per_gate=3, post=1, pre=2, eps=EPS)
    h, y = hif4.hif4_block_norm(x, w, b, residual=r, gate=gate, post_weight=wp, **kw)
    (_, xs), (_, rs), (_, gs) = strided(x, 16), strided(r, 32), strided(gate, 48)
    (hw, hs), (yw, ys) = strided(torch.full_like(x, 7.0), 24), strided(torch.full_like(x, 7.0), 40)
    hif4.hif4_block_norm(xs, w, b, residual=rs, gate=gs, post_weight=wp, out_h=hs, out_y=ys, **kw)
    assert torch.equal(hs, h) and torch.equal(ys, y)
    for t, v in ((hw, hs), (yw, ys)):
        v.fill_(7.0)
        assert (t == 7.0).all(), "written outside the matrix"
    check_forward(hif4, x, r, gate, wp.float(), w.float(), b.float(), 0.5, 3, 1, 2, "FP32 weights")
    alone, none = hif4.hif4_block_norm(x, residual=r, gate=gate, post_weight=wp, **dict(kw, pre=0))
    size = h.double().abs()
    mag = size + (0.5 * r.double()).abs() + x.double().abs().amax(1, keepdim=True)
    assert none is None and bool(((alone.double() - h.double()).abs() <= 2.1 * (U[dtype] * size + ARITH * mag + TINY[dtype])).all())
    plain, none = hif4.hif4_block_norm(x, residual=r, res_scale=0.5, pre=0)
    assert none is None and torch.equal(plain, (0.5 * r.float() + x.float()).to(dtype))
    for target in ("x", "r"):
        x2, r2 = x.clone(), r.clone()
        h2, y2 = hif4.hif4_block_norm(x2, w, b, residual=r2, gate=gate, post_weight=wp, out_h=x2 if target == "x" else r2, **kw)
        assert torch.equal(h2, h) and torch.equal(y2, y)


# rows a block: 10 (four blocks an SM, eight for the plain norm), 8 (two, plain) or 16, 10 (one), 10 (one), 4 (one)
GRADIENT = [(6000, 1024), (2500, 4096), (1500, 5120), (1500, 8192), (700, 10240)]
GRADIENT_KINDS = [(0, 1, 0), (0, 2, 0), (1, 1, 0), (1, 1, 7), (2, 2, 600), (0, 2, 5), (1, 2, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", GRADIENT)
@pytest.mark.parametrize("post,pre,rpg", GRADIENT_KINDS)
def test_gradients(hif4, dtype, rows, cols, post, pre, rpg):
    check_gradients(hif4, dtype, rows, cols, post, pre, rpg)
    assert hif4.hif4_last_device_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(6000, 1024), (1500, 5120)])
def test_gradient_strides_and_weight_types(hif4, dtype, rows, cols):
    x, r, gate, wp, w, b = make(rows, cols, dtype, dtype, 1, 1, 3, True, 19)
    dy, dh = (torch.randn(rows, cols, device="cuda").to(dtype) for _ in range(2))
    kw = dict(res_scale=0.5, rows_per_gate=3, post=1, pre=1, eps=EPS)
    want = hif4.hif4_block_norm_backward(dy, r, w, dh=dh, x=x, gate=gate, post_weight=wp, **kw)
    s = [strided(t, 16 * (i + 1))[1] for i, t in enumerate((dy, r, dh, x, gate))]
    got = hif4.hif4_block_norm_backward(s[0], s[1], w, dh=s[2], x=s[3], gate=s[4], post_weight=wp, **kw)
    wide = hif4.hif4_block_norm_backward(dy, r, w.float(), dh=dh, x=x, gate=gate, post_weight=wp.float(), **kw)
    for k, v in want.items():
        if v is not None:
            assert torch.equal(got[k], v) and torch.equal(wide[k], v), k


@pytest.mark.parametrize("dtype,rows,cols", [(t, 6000, 1024) for t in TYPES] + [(t, 1500, 5120) for t in TYPES[:2]])
def test_absent_gradients_are_zeros(hif4, dtype, rows, cols):
    x, r, gate, wp, w, b = make(rows, cols, dtype, dtype, 1, 1, 3, True, 19)
    dy, dh = (torch.randn(rows, cols, device="cuda").to(dtype) for _ in range(2))
    kw = dict(res_scale=0.5, rows_per_gate=3, post=1, pre=1, eps=EPS)
    zero = torch.zeros_like(x)
    a = hif4.hif4_block_norm_backward(dy, r, w, x=x, gate=gate, post_weight=wp, **kw)
    z = hif4.hif4_block_norm_backward(dy, r, w, dh=zero, x=x, gate=gate, post_weight=wp, **kw)
    a2 = hif4.hif4_block_norm_backward(None, None, None, dh=dh, x=x, gate=gate, post_weight=wp, **kw)
    z2 = hif4.hif4_block_norm_backward(zero, r, w, dh=dh, x=x, gate=gate, post_weight=wp, **kw)
    for got, ref, keys in ((a, z, ("dx", "dresidual", "dgate", "dweight", "dpost_weight")), (a2, z2, ("dx", "dresidual", "dgate", "dpost_weight"))):
        for k in keys:
            assert torch.equal(got[k], ref[k]), k
