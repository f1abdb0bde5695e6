"""What the native calls do with arguments that are not what they should be, and with outputs that are not wanted."""
import pytest
import torch

from tests.test_gpu_block_norm import hif4, make  # noqa: F401
from tests.test_gpu_linear_act import operands

pytestmark = pytest.mark.gpu


def test_codes_past_32_bits_are_refused(hif4):
    """2^32 + 1 is no code of a norm, an activation or a rounding, and not the code 1 either."""
    x, r, gate, wp, w, b = make(4, 128, torch.bfloat16, torch.bfloat16, 1, 1, 0, True, 1)
    far = 2 ** 32
    xl, wl, bl = operands(hif4, 4, 64, 256, torch.bfloat16, True, 3)
    dy = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    for f in (lambda: hif4.hif4_block_norm(x, w, pre=far + 1), lambda: hif4.hif4_block_norm(x, w, post=far + 1),
              lambda: hif4.hif4_block_norm(x, w, mode=far), lambda: hif4.hif4_block_norm_backward(x, x, w, pre=far + 1),
              lambda: hif4.hif4_block_norm_backward(x, x, w, x=x, post=far + 1),
              lambda: hif4.hif4_linear_act(xl, wl[0], act=far + 2), lambda: hif4.hif4_linear_act(xl, wl[0], mode=far),
              lambda: hif4.hif4_gated_linear(xl, *wl, act=far + 2), lambda: hif4.hif4_linear_act_backward(dy, xl, wl[0], act=far + 2),
              lambda: hif4.hif4_gated_linear_backward(dy, xl, *wl, mode=far)):
        with pytest.raises(hif4.Hif4Error) as e:
            f()
        assert e.value.code == 4


def test_a_flag_that_is_neither_true_nor_false(hif4):
    x = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    two = torch.ones(2)
    for f in (lambda: hif4.hif4_block_norm(x, None, units=two), lambda: hif4.hif4_block_norm_backward(x, x, None, want_dresidual=two)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            f()


def test_one_row_of_gates_for_any_number_of_rows(hif4):
    x, r, gate, wp, w, b = make(50, 320, torch.bfloat16, torch.bfloat16, 1, 1, 50, True, 1)
    kw = dict(gate=gate, post=1, post_weight=wp)
    want = hif4.hif4_block_norm(x, w, residual=r, rows_per_gate=50, **kw)
    dwant = hif4.hif4_block_norm_backward(x, want[0], w, dh=r, x=x, rows_per_gate=50, **kw)
    for per in (51, 2 ** 31, 2 ** 63 - 1):
        got = hif4.hif4_block_norm(x, w, residual=r, rows_per_gate=per, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        d = hif4.hif4_block_norm_backward(x, want[0], w, dh=r, x=x, rows_per_gate=per, **kw)
        assert all(torch.equal(d[k], v) for k, v in dwant.items() if v is not None)


def test_a_workspace_is_as_large_as_its_memory(hif4):
    """An expanded tensor counts more elements than it holds: it is no workspace."""
    x, w, b = operands(hif4, 64, 256, 512, torch.bfloat16, False, 3)
    dy = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")
    n = torch.zeros(512, 512, dtype=torch.bfloat16, device="cuda")
    expanded = torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 28)
    before = hif4.launch_count()
    for f in (lambda: hif4.hif4_linear_act(x, w[0], workspace=expanded), lambda: hif4.hif4_linear_act_backward(dy, x, w[0], act=2, workspace=expanded),
              lambda: hif4.hif4_block_norm_backward(n, n, None, workspace=expanded)):
        with pytest.raises(ValueError):
            f()
    assert hif4.launch_count() == before
    space = torch.empty(1 << 26, dtype=torch.float32, device="cuda")
    assert torch.equal(hif4.hif4_linear_act(x, w[0], workspace=space), hif4.hif4_linear_act(x, w[0]))


@pytest.mark.parametrize("rows,cols", [(90, 320), (70, 1001), (700, 4096), (400, 10240)])
@pytest.mark.parametrize("post,pre,rpg", [(0, 1, 0), (1, 1, 7), (2, 2, 0), (0, 2, 5)])
def test_norm_gradients_that_are_not_wanted(hif4, rows, cols, post, pre, rpg):
    """Each can be declined; the others keep their bits."""
    x, r, gate, wp, w, b = make(rows, cols, torch.bfloat16, torch.bfloat16, post, pre, rpg, True, 3)
    f = lambda **kw: hif4.hif4_block_norm_backward(x, r, w, dh=r, x=x, bias=b is not None, gate=gate, rows_per_gate=rpg, post=post,    # noqa: E731
                                                   post_weight=wp, pre=pre, **kw)
    full = f()
    of = {"dx": "dx", "dresidual": "dresidual", "dgate": "dgate", "dweight": "dweights", "dbias": "dweights", "dpost_weight": "dweights"}
    wants = ["dx", "dresidual", "dgate", "dweights"]
    for off in [[k] for k in wants] + [[k for k in wants if k != keep] for keep in wants] + [wants]:
        got = f(**{"want_" + k: False for k in off})
        for k, v in full.items():
            if v is None or of[k] in off:
                assert got[k] is None, (off, k)
            else:
                assert torch.equal(got[k], v), (off, k)
