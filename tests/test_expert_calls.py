"""Argument errors of routing, experts' rows and 4-bit block formats: found on the host, without a device.  No GPU."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64, ci, vp, cf, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
OK, NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED = 0, 1, 2, 3, 4, 8
P = 0x10000                                              # an aligned address that nothing reads


class Route(ctypes.Structure):
    _fields_ = [("tokens", i64), ("experts", i64), ("top_k", i64), ("logits", vp), ("dt", ci), ("ld_logits", i64), ("bias", vp), ("score", ci),
                ("groups", i64), ("top_groups", i64), ("group_best", i64), ("renormalize", ci), ("scale", cf), ("ids", vp), ("weights", vp)]


class RouteBackward(ctypes.Structure):
    _fields_ = [("tokens", i64), ("experts", i64), ("top_k", i64), ("logits", vp), ("dt", ci), ("ld_logits", i64), ("ids", vp), ("dweights", vp),
                ("score", ci), ("renormalize", ci), ("scale", cf), ("dlogits", vp), ("ld_dlogits", i64)]


class Dispatch(ctypes.Structure):
    _fields_ = [("tokens", i64), ("cols", i64), ("top_k", i64), ("rows", i64), ("x", vp), ("dt", ci), ("ld_x", i64), ("row_of", vp), ("kind", ci),
                ("mode", ci), ("gain", vp), ("out", vp), ("ld_out", i64), ("out_scales", vp)]


class Combine(ctypes.Structure):
    _fields_ = [("tokens", i64), ("cols", i64), ("top_k", i64), ("rows", i64), ("in_", vp), ("dt_in", ci), ("ld_in", i64), ("row_of", vp),
                ("weights", vp), ("dt", ci), ("residual", vp), ("ld_residual", i64), ("res_scale", cf), ("y", vp), ("ld_y", i64)]


class CombineBackward(ctypes.Structure):
    _fields_ = [("tokens", i64), ("cols", i64), ("top_k", i64), ("rows", i64), ("dy", vp), ("dt", ci), ("ld_dy", i64), ("row_of", vp),
                ("weights", vp), ("in_", vp), ("dt_in", ci), ("ld_in", i64), ("din", vp), ("ld_din", i64), ("dweights", vp)]


class Gemm(ctypes.Structure):
    _fields_ = [("M", i64), ("N", i64), ("K", i64), ("fmt", ci), ("A_codes", vp), ("A_scales", vp), ("B_codes", vp), ("B_scales", vp),
                ("alpha", vp), ("dt", ci), ("Y", vp), ("ld_y", i64), ("num_groups", ci), ("group_offsets", vp)]


@pytest.fixture(scope="module")
def lib():
    import paper_2602_11287_b200 as hif4
    return hif4.lib


def call(lib, name, args, **fields):
    f = getattr(lib, name)
    f.restype = ci
    return f(ctypes.byref(args(**fields)), None)


def test_structures_are_the_header_s(tmp_path):
    """Sizes as a C program sees them, so that the fields above lie where the library reads them."""
    names = {"hif4_route_args": Route, "hif4_route_backward_args": RouteBackward, "hif4_dispatch_args": Dispatch, "hif4_combine_args": Combine,
             "hif4_combine_backward_args": CombineBackward, "hif4_bfp4_gemm_args": Gemm}
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "hif4.h"\nint main(void) {\n' + "".join(f'  printf("{n} %zu\\n", sizeof({n}));\n' for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        n, size = line.split()
        assert ctypes.sizeof(names[n]) == int(size), n


def test_route(lib):
    good = dict(tokens=4, experts=64, top_k=2, logits=P, dt=1, ld_logits=64, score=0, groups=8, top_groups=2, group_best=2, renormalize=1, scale=1.0,
                ids=P, weights=P)
    for change, want in ((dict(tokens=-1), SHAPE), (dict(experts=0), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=65), SHAPE), (dict(top_k=17), SHAPE),
                         (dict(ld_logits=63), SHAPE), (dict(dt=3), DTYPE), (dict(score=2), DTYPE), (dict(groups=5), SHAPE), (dict(groups=0), SHAPE),
                         (dict(top_groups=0), SHAPE), (dict(top_groups=9), SHAPE), (dict(group_best=0), SHAPE), (dict(group_best=3), SHAPE),
                         (dict(groups=64, top_groups=64), SHAPE), (dict(groups=64, top_groups=64, group_best=1), UNSUPPORTED),
                         (dict(experts=2048, ld_logits=2048), UNSUPPORTED), (dict(groups=1, top_groups=1, top_k=33), UNSUPPORTED), (dict(logits=None), NULL),
                         (dict(ids=None), NULL), (dict(weights=None), NULL), (dict(logits=P + 2), ALIGN), (dict(ids=P + 1), ALIGN),
                         (dict(bias=P + 2), ALIGN), (dict(tokens=0, logits=None, ids=None, weights=None), OK)):
        assert call(lib, "hif4_route", Route, **{**good, **change}) == want, change
    lib.hif4_route.restype = ci
    assert lib.hif4_route(None, None) == NULL
    good = dict(tokens=4, experts=64, top_k=2, logits=P, dt=0, ld_logits=64, ids=P, dweights=P, score=1, renormalize=1, scale=1.0, dlogits=P, ld_dlogits=64)
    for change, want in ((dict(ld_dlogits=63), SHAPE), (dict(dlogits=None), NULL), (dict(dweights=None), NULL), (dict(dt=7), DTYPE), (dict(dlogits=P + 1), ALIGN),
                         (dict(experts=1025, ld_logits=1025, ld_dlogits=1025), UNSUPPORTED), (dict(tokens=0, dlogits=None), OK)):
        assert call(lib, "hif4_route_backward", RouteBackward, **{**good, **change}) == want, change


def test_plan(lib):
    n = sz(5)
    ask = lambda t, k, e: lib.hif4_expert_plan_workspace(t, k, e, ctypes.byref(n))      # noqa: E731
    assert ask(256, 8, 256) == OK and n.value == 0                   # 2048 assignments: one block
    assert ask(257, 8, 256) == OK and n.value == 2 * 256 * 4         # two blocks' counts
    assert ask(1 << 20, 1, 100) == OK and n.value == (256 * 100 * 4 + 255) // 256 * 256      # 256 blocks at most
    assert ask(-1, 8, 4) == SHAPE and ask(1, 0, 4) == SHAPE and ask(1, 1, 0) == SHAPE and ask(1 << 31, 1, 4) == SHAPE and ask(1 << 62, 1 << 62, 4) == SHAPE
    assert ask(1, 1, 1025) == UNSUPPORTED and lib.hif4_expert_plan_workspace(1, 1, 1, None) == NULL
    f = lib.hif4_expert_plan
    f.restype = ci
    f.argtypes = [vp, i64, i64, i64, vp, vp, vp, sz, vp]
    assert f(P, 1000, 8, 256, P, P, None, 0, None) == NULL and f(P, 1000, 8, 256, P, P, P, 8, None) == 5
    assert f(P, 1000, 8, 256, P, P, P + 16, 1 << 20, None) == ALIGN and f(P, 10, 8, 256, P + 4, P, None, 0, None) == ALIGN
    assert f(None, 10, 8, 256, P, P, None, 0, None) == NULL and f(P, 10, 8, 256, None, P, None, 0, None) == NULL


def test_dispatch_and_combine(lib):
    good = dict(tokens=4, cols=128, top_k=2, rows=8, x=P, dt=0, ld_x=128, row_of=P, kind=0, mode=0, out=P, ld_out=128, out_scales=P)
    for change, want in ((dict(kind=4), DTYPE), (dict(kind=-1), DTYPE), (dict(kind=1, mode=2), DTYPE), (dict(dt=5), DTYPE), (dict(ld_x=127), SHAPE),
                         (dict(ld_out=127), SHAPE), (dict(kind=1, cols=100), SHAPE), (dict(kind=2, out_scales=None), NULL), (dict(out=None), NULL),
                         (dict(row_of=None), NULL), (dict(x=None), NULL), (dict(kind=1, x=P + 2), ALIGN), (dict(kind=2, ld_x=129), ALIGN),
                         (dict(kind=3, out=P + 8), ALIGN), (dict(kind=3, gain=P + 2), ALIGN), (dict(x=P + 1), ALIGN), (dict(rows=-1), SHAPE),
                         (dict(rows=1 << 31), SHAPE), (dict(top_k=0), SHAPE), (dict(tokens=1 << 31), SHAPE), (dict(tokens=0, x=None), OK),
                         (dict(rows=0, out=None), OK)):
        assert call(lib, "hif4_dispatch", Dispatch, **{**good, **change}) == want, change
    good = dict(tokens=4, cols=128, top_k=2, rows=8, in_=P, dt_in=1, ld_in=128, row_of=P, dt=0, res_scale=1.0, y=P, ld_y=128)
    for change, want in ((dict(dt=3), DTYPE), (dict(dt_in=-1), DTYPE), (dict(ld_in=1), SHAPE), (dict(ld_y=1), SHAPE), (dict(residual=P, ld_residual=1), SHAPE),
                         (dict(in_=None), NULL), (dict(y=None), NULL), (dict(in_=P + 2), ALIGN), (dict(y=P + 1), ALIGN), (dict(weights=P + 2), ALIGN),
                         (dict(cols=0), OK), (dict(tokens=0), OK)):
        assert call(lib, "hif4_combine", Combine, **{**good, **change}) == want, change
    good = dict(tokens=4, cols=128, top_k=2, rows=8, dy=P, dt=0, ld_dy=128, row_of=P, in_=P, dt_in=1, ld_in=128, din=P, ld_din=128, dweights=P)
    for change, want in ((dict(ld_dy=1), SHAPE), (dict(ld_din=1), SHAPE), (dict(ld_in=1), SHAPE), (dict(in_=None), NULL), (dict(dy=None), NULL),
                         (dict(din=P + 2), ALIGN), (dict(din=None, dweights=None, dy=None), OK), (dict(tokens=0), OK)):
        assert call(lib, "hif4_combine_backward", CombineBackward, **{**good, **change}) == want, change


def test_block_formats(lib):
    size = lib.hif4_bfp4_scale_bytes
    assert size(3, 64, 2) == 48 and size(3, 256, 2) == 48 and size(3, 320, 2) == 96 and size(3, 320, 1) == 48 and size(3, 576, 1) == 96
    assert size(3, 100, 2) == 0 and size(-1, 64, 2) == 0 and size(3, 64, 0) == 0 and size(3, 64, 3) == 0
    for name in ("hif4_bfp4_quantize", "hif4_bfp4_quantize_transposed"):
        f = getattr(lib, name)
        f.restype = ci
        f.argtypes = [vp, ci, i64, i64, i64, ci, vp, vp, vp, vp]
        assert f(P, 0, 100, 100, 100, 2, None, P, P, None) == SHAPE and f(P, 0, 64, 128, 64, 2, None, P, P, None) == SHAPE
        assert f(P, 9, 64, 128, 128, 2, None, P, P, None) == DTYPE and f(P, 0, 64, 128, 128, 3, None, P, P, None) == DTYPE
        assert f(None, 0, 64, 128, 128, 2, None, P, P, None) == NULL and f(P + 2, 0, 64, 128, 128, 2, None, P, P, None) == ALIGN
        assert f(P, 0, 64, 128, 129, 2, None, P, P, None) == ALIGN and f(P, 0, 64, 128, 128, 1, P + 2, P, P, None) == ALIGN
        assert f(P, 0, 64 << 31, 64 << 31, 64 << 31, 1, None, P, P, None) == SHAPE and f(None, 0, 0, 128, 128, 1, None, None, None, None) == OK
    f = lib.hif4_bfp4_dequantize
    f.restype = ci
    f.argtypes = [vp, vp, i64, i64, ci, vp, vp, ci, i64, vp]
    assert f(P, P, 4, 64, 2, None, P, 2, 64, None) == DTYPE and f(P, P, 4, 64, 0, None, P, 0, 64, None) == DTYPE and f(P, P, 4, 60, 2, None, P, 0, 64, None) == SHAPE
    good = dict(M=4, N=8, K=128, fmt=2, A_codes=P, A_scales=P, B_codes=P, B_scales=P, dt=0, Y=P, ld_y=8)
    for name, more in (("hif4_bfp4_gemm", {}), ("hif4_bfp4_grouped_gemm", dict(num_groups=2, group_offsets=P))):
        for change, want in ((dict(K=0), SHAPE), (dict(K=100), SHAPE), (dict(M=-1), SHAPE), (dict(ld_y=7), SHAPE), (dict(M=1 << 31), SHAPE), (dict(fmt=0), DTYPE),
                             (dict(fmt=3), DTYPE), (dict(dt=4), DTYPE), (dict(Y=None), NULL), (dict(B_scales=None), NULL), (dict(A_codes=P + 8), ALIGN),
                             (dict(alpha=P + 2), ALIGN), (dict(Y=P + 1), ALIGN), (dict(M=0, Y=None), OK), (dict(N=0, ld_y=0), OK)):
            assert call(lib, name, Gemm, **{**good, **more, **change}) == want, (name, change)
    assert call(lib, "hif4_bfp4_grouped_gemm", Gemm, **good, num_groups=-1, group_offsets=P) == SHAPE
    assert call(lib, "hif4_bfp4_grouped_gemm", Gemm, **good, num_groups=2) == NULL
    assert call(lib, "hif4_bfp4_grouped_gemm", Gemm, **{**good, "N": 1 << 20, "ld_y": 1 << 20}, num_groups=1 << 20, group_offsets=P) == SHAPE
    assert call(lib, "hif4_bfp4_grouped_gemm", Gemm, **good, num_groups=0) == OK


def test_limits_of_the_header_are_stated_once():
    text = open(os.path.join(ROOT, "include", "hif4.h")).read()
    assert re.search(r"HIF4_ROUTE_MAX_EXPERTS 1024\b", text) and re.search(r"HIF4_ROUTE_MAX_TOP_K 32\b", text) and re.search(r"HIF4_ROUTE_MAX_GROUPS 32\b", text)
