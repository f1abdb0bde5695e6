"""include/hif4.h as a C program sees it.  No GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "hif4.h"\nint main(void) { hif4_block_norm_args a; hif4_linear_act_args b; return sizeof(a) == sizeof(b); }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "h.o")], check=True)


def test_argument_errors_of_the_block_calls_need_no_device():
    """Null arguments, sizes, types and workspaces are refused on the host; empty sizes are answered there."""
    import ctypes

    import paper_2602_11287_b200 as hif4
    lib = hif4.lib
    n = ctypes.c_size_t(7)
    assert lib.hif4_block_norm_backward_workspace(10, 4096, ctypes.byref(n)) == 0
    assert n.value == 5 * 10 * 4096 * 4                              # ten blocks of a row each, five planes of column sums
    assert lib.hif4_block_norm_backward_workspace(10, 40000, ctypes.byref(n)) == 2
    assert lib.hif4_block_norm_backward_workspace(10, 64, None) == 1
    for name in ("hif4_block_norm", "hif4_linear_act", "hif4_gated_linear", "hif4_linear_act_backward", "hif4_gated_linear_backward"):
        call = getattr(lib, name)
        call.restype = ctypes.c_int
        if name == "hif4_block_norm":
            assert call(None, None) == 1
        else:
            assert call(None, None, ctypes.c_size_t(0), None) == 1
