"""MXFP4 and NVFP4: infinite gains, single rows with any stride."""
import math

import pytest
import torch

from tests import bfp4_reference as ref
from tests.test_gpu_bfp4 import MX, NV, gen, hif4, matrix  # noqa: F401  (hif4: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("gain", [math.inf, -math.inf])
def test_infinite_gains(hif4, fmt, dtype, gain):  # noqa: F811
    """Zeros become NaN and the others infinite: blocks with zeros are NaN blocks, wherever they are converted, the rest saturates."""
    x = matrix(128, 320, dtype, 12)
    x[64:] = torch.where(x[64:] == 0, 1.0, x[64:].float()).to(dtype)      # half of the blocks have no zeros
    x[:, 64:128] = torch.where(x[:, 64:128] == 0, -2.0, x[:, 64:128].float()).to(dtype)
    g = torch.full((1,), gain, device="cuda")
    want = ref.pack(*ref.convert(x, fmt, g))
    bad = 255 if fmt == MX else 127
    used = want[1].transpose(0, 1).reshape(128, -1)[:, : 320 // ref.BLOCK[fmt]]
    assert bool((used == bad).any()) and bool((used != bad).any())
    got = hif4.hif4_bfp4_quantize(x, fmt, gain=g)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    down = hif4.hif4_bfp4_quantize_transposed(x.t().contiguous()[:, :128], fmt, gain=g)
    assert torch.equal(down[0], want[0]) and torch.equal(down[1], want[1])
    row_of = torch.arange(128, dtype=torch.int32, device="cuda").flip(0).view(128, 1).contiguous()
    rows = hif4.hif4_dispatch(x, row_of, fmt=fmt, gain=g)
    assert torch.equal(rows[0].flip(0), want[0]) and torch.equal(rows[1].flip(1), want[1])
    for dt in (torch.bfloat16, torch.float32):
        back, v = hif4.hif4_bfp4_dequantize(got, fmt, dt, gain=g), (ref.values(*want, fmt).float() / g).to(dt)
        assert torch.equal(back.isnan(), v.isnan()) and torch.equal(back.nan_to_num(0.0), v.nan_to_num(0.0))


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_one_row_with_any_stride(hif4, fmt, dtype):  # noqa: F811
    """A row of its own has no next one: only its address has to be a multiple of 16 bytes."""
    x = matrix(5, 321, dtype, 13)
    row = x.view(-1)[: 5 * 321].view(5, 321)[:1, :320]
    assert row.stride(0) == 321 and row.data_ptr() % 16 == 0
    alone = row.flatten().clone().view(1, 320)              # the same row in a matrix of its own
    want = hif4.hif4_bfp4_quantize(alone, fmt)
    got = hif4.hif4_bfp4_quantize(row, fmt)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out_type = torch.float32 if dtype == torch.float32 else torch.bfloat16
    wide = torch.full((2, 321), 7.0, dtype=out_type, device="cuda")
    hif4.hif4_bfp4_dequantize(got, fmt, out=wide[:1, :320])
    assert torch.equal(wide[:1, :320], hif4.hif4_bfp4_dequantize(got, fmt, out_type)) and bool((wide.view(-1)[320:] == 7.0).all())
    row_of = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    rows = hif4.hif4_dispatch(row, row_of, fmt=fmt)
    assert torch.equal(rows[0], want[0].expand(2, -1)) and torch.equal(rows[1], want[1].expand(-1, 2, -1))
    units = hif4.hif4_dispatch(row, row_of, fmt=hif4.HIF4_FMT_HIF4)
    assert torch.equal(units, hif4.hif4_quantize(alone).expand(2, -1, -1))
