"""stream=: what a call of the HiF4 format allocates belongs to that stream, so that no pending work of another one writes to it."""
import pytest
import torch

from tests.test_gpu_experts import gen, hif4  # noqa: F401  (hif4: fixture)

pytestmark = pytest.mark.gpu


def calls(h):
    g = gen(1)
    x = torch.randn(512, 512, generator=g, device="cuda").to(torch.bfloat16)
    u = h.hif4_quantize(x)
    off, few, two = torch.tensor([0, 100, 512], device="cuda"), u[:40].contiguous(), torch.stack([u, u])
    return {"quantize": lambda s: h.hif4_quantize(x, stream=s), "quantize_transposed": lambda s: h.hif4_quantize_transposed(x, stream=s),
            "dequantize": lambda s: h.hif4_dequantize(u, stream=s), "gemm": lambda s: h.hif4_gemm(u, u, stream=s),
            "few_rows": lambda s: h.hif4_gemm(few, u, stream=s), "linear": lambda s: h.hif4_linear(x, u, stream=s),
            "one_token": lambda s: h.hif4_linear(x[:1], u, stream=s),
            "grouped": lambda s: h.hif4_grouped_gemm(u, two, off, stream=s), "mse": lambda s: h.hif4_mse_roundtrip(x, 2, stream=s)[0]}


@pytest.mark.parametrize("name", ["quantize", "quantize_transposed", "dequantize", "gemm", "few_rows", "linear", "one_token", "grouped", "mse"])
def test_outputs_are_the_stream_s(hif4, name):  # noqa: F811
    f = calls(hif4)[name]
    want = f(None)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        f(None)                                             # (memory of its own)
    busy = torch.empty(1 << 28, device="cuda")
    torch.cuda.synchronize()
    blocks = [torch.empty_like(want) for _ in range(8)]
    for _ in range(20):
        busy.normal_()                                      # some milliseconds of work before the blocks are written
    for b in blocks:
        b.fill_(77)
    del blocks, b                                           # free for this stream's next calls, which come after that
    got = f(side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_two_streams_at_once(hif4):  # noqa: F811
    """Eager calls on two streams, with workspaces of their own: the same bits as one after the other."""
    fs = calls(hif4)
    want = {n: f(None) for n, f in fs.items()}
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [(n, f(st)) for _ in range(3) for n, f in fs.items() for st in streams]
    torch.cuda.synchronize()
    for n, v in got:
        assert torch.equal(v, want[n]), n
