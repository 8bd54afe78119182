"""The gated block layers' part of the C ABI: struct layouts and constants agree
between the header and the binding, and host-side checks refuse bad calls before
anything touches the GPU (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_32415_gb300 import _lib, build
    build.build()
    return _lib.load()


def test_struct_layouts_and_constants_match_c(tmp_path):
    from paper_2609_32415_gb300 import _lib
    structs = {"ra_rope_tensor": _lib.RaRopeTensor, "ra_rope_args": _lib.RaRopeArgs, "ra_resnorm_seg": _lib.RaResnormSeg,
               "ra_resnorm_args": _lib.RaResnormArgs, "ra_resnorm_grad_args": _lib.RaResnormGradArgs,
               "ra_glu_seg": _lib.RaGluSeg, "ra_glu_args": _lib.RaGluArgs, "ra_glu_grad_args": _lib.RaGluGradArgs}
    lines, want = [], []
    for name, cls in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for field, *_ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field))
            want.append(getattr(cls, field).offset)
    for c in ("RA_NORM_NONE", "RA_NORM_LAYER", "RA_NORM_RMS", "RA_ACT_SILU", "RA_ACT_GELU"):
        lines.append('printf("%%d\\n", (int)%s);' % c)
        want.append(getattr(_lib, c))
    src = tmp_path / "layout_gated.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"refadapt.h\"\nint main(void) {\n%s\nreturn 0;\n}\n"
                   % "\n".join(lines))
    exe = tmp_path / "layout_gated"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == want


def refused(lib, status, text):
    from paper_2609_32415_gb300._lib import RA_EINVAL
    assert status == RA_EINVAL and text in lib.refadapt_last_error(), lib.refadapt_last_error()


def test_rope_axes_refuses_before_launch(lib):
    from paper_2609_32415_gb300 import _lib
    refused(lib, lib.refadapt_rope_axes(None, None), b"args is NULL")
    a = _lib.RaRopeArgs()
    a.B, a.n, a.d, a.n_axes, a.base, a.n_tensors, a.pos = 1, 4, 64, 2, 1e4, 1, 0x40000
    a.axis_dim[0], a.axis_dim[1] = 32, 32
    for i in range(2):
        a.t[i].heads = 2
        a.t[i].x = a.t[i].out = _lib.RaSeg(0x10000, 512, 256, 64, 4, 0)
    for field, value, text in (("d", 60, b"multiple of 8"), ("d", 264, b"256"), ("n_tensors", 3, b"tensors"),
                               ("n_axes", 5, b"axes"), ("inverse", 2, b"inverse"), ("B", 0, b"B >= 1"),
                               ("base", float("inf"), b"base"), ("n", 5, b"rows differ"), ("pos", 0, b"pos NULL"),
                               ("pos_stride_s", -1, b"pos_stride_s")):
        keep = getattr(a, field)
        setattr(a, field, value)
        refused(lib, lib.refadapt_rope_axes(ctypes.byref(a), None), text)
        setattr(a, field, keep)
    a.axis_dim[1] = 34
    refused(lib, lib.refadapt_rope_axes(ctypes.byref(a), None), b"66 columns")
    dims = (ctypes.c_int32 * 2)(32, 31)
    refused(lib, lib.refadapt_rope_axes_table(0x10000, 0x20000, 4, 64, 2, dims, 1e4, None), b"even")
    refused(lib, lib.refadapt_rope_axes_table(0x10004, 0x20000, 4, 64, 2, dims, 1e4, None), b"misaligned")


def test_residual_norm_refuses_before_launch(lib):
    from paper_2609_32415_gb300 import _lib
    refused(lib, lib.refadapt_residual_norm(None, None), b"args is NULL")
    a = _lib.RaResnormArgs()
    a.B, a.C, a.n_seg, a.post, a.pre, a.eps, a.alpha = 2, 64, 1, 2, 1, 1e-6, 1.0
    s = a.seg[0]
    s.rows = 4
    for n, p in (("h", 0x10000), ("y", 0x20000), ("h_out", 0x30000), ("x", 0x40000)):
        setattr(s, n, p)
        setattr(s, n + "_stride_s", 256)
        setattr(s, n + "_stride_r", 64)
    for field, value, text in (("C", 60, b"multiple of 8"), ("C", 5128, b"5120"), ("n_seg", 4, b"n_seg"),
                               ("post", 3, b"known norms"), ("pre", -1, b"known norms"), ("B", 0, b"B >= 1")):
        keep = getattr(a, field)
        setattr(a, field, value)
        refused(lib, lib.refadapt_residual_norm(ctypes.byref(a), None), text)
        setattr(a, field, keep)
    for field, value, text in (("rows", -1, b"rows < 0"), ("gated", 1, b"mode is NULL"), ("h", 0, b"h is NULL"),
                               ("y", 0x20008, b"y must"), ("x_stride_r", 56, b"x must"), ("h_out_stride_s", 0, b"h_out"),
                               ("gate", 0x50004, b"gate"), ("pre_w", 0x50004, b"pre_w"), ("x", 0x30000, b"same tensor"),
                               ("rows", 1 << 29, b"too many rows")):
        keep = getattr(s, field)
        setattr(s, field, value)
        refused(lib, lib.refadapt_residual_norm(ctypes.byref(a), None), text)
        setattr(s, field, keep)
    s.x, s.x_stride_r = 0x10000, 72  # in place with another stride
    refused(lib, lib.refadapt_residual_norm(ctypes.byref(a), None), b"in place")
    assert lib.refadapt_residual_norm_backward_workspace_size(0, 4, 64) == 0
    assert lib.refadapt_residual_norm_backward_workspace_size(2, 4, 64) >= 2 * 3 * 64 * 4
    refused(lib, lib.refadapt_residual_norm_backward(None, None), b"args is NULL")


def test_glu_refuses_before_launch(lib):
    from paper_2609_32415_gb300 import _lib
    refused(lib, lib.refadapt_glu(None, None), b"args is NULL")
    a = _lib.RaGluArgs()
    a.B, a.F, a.C, a.act, a.n_seg = 2, 128, 64, 0, 1
    s = a.seg[0]
    s.rows, s.w_gate, s.w_up = 4, 0x50000, 0x60000
    for n, p, width in (("x", 0x10000, 64), ("out", 0x20000, 128), ("pre_gate", 0x30000, 128), ("pre_up", 0x40000, 128)):
        setattr(s, n, p)
        setattr(s, n + "_stride_s", 4 * width)
        setattr(s, n + "_stride_r", width)
    for field, value, text in (("C", 60, b"multiples of 8"), ("F", 56, b"at least 64"), ("act", 2, b"activation"),
                               ("n_seg", 0, b"n_seg"), ("B", 0, b"B >= 1")):
        keep = getattr(a, field)
        setattr(a, field, value)
        refused(lib, lib.refadapt_glu(ctypes.byref(a), None), text)
        setattr(a, field, keep)
    for field, value, text in (("rows", -1, b"rows < 0"), ("gated", 1, b"mode is NULL"), ("w_up", 0x60008, b"w_up"),
                               ("pre_up", 0, b"go together"), ("x", 0, b"x must"), ("out_stride_r", 120, b"out must"),
                               ("out_stride_s", 0, b"out must"), ("rows", 1 << 29, b"too many rows")):
        keep = getattr(s, field)
        setattr(s, field, value)
        refused(lib, lib.refadapt_glu(ctypes.byref(a), None), text)
        setattr(s, field, keep)
    refused(lib, lib.refadapt_glu_backward(None, None), b"args is NULL")
    b = _lib.RaGluGradArgs()
    b.B, b.rows, b.C, b.F, b.O = 1, 4, 64, 128, 64
    refused(lib, lib.refadapt_glu_backward(ctypes.byref(b), None), b"no gradient")
    b.dx, b.dw_up = 0x10000, 0x20004
    refused(lib, lib.refadapt_glu_backward(ctypes.byref(b), None), b"16-byte aligned")
    assert lib.refadapt_glu_backward_workspace_size(1, 4, 64, 128, 64) >= 2 * 4 * 128 * 2
    assert lib.refadapt_glu_backward_workspace_size(1, -1, 64, 128, 64) == 0
