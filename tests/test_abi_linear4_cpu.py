"""The 4-bit layers' and the optimiser's part of the C ABI: struct layouts and constants
agree between the header and the binding, and host-side checks refuse bad calls before
anything touches the GPU (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

from test_abi_layers_cpu import refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_32415_gb300 import _lib, build
    build.build()
    return _lib.load()


def test_struct_layouts_and_constants_match_c(tmp_path):
    from paper_2609_32415_gb300 import _lib
    structs = {"ra_quant4_seg": _lib.RaQuant4Seg, "ra_quant4_args": _lib.RaQuant4Args, "ra_gemm4_seg": _lib.RaGemm4Seg,
               "ra_gemm4_args": _lib.RaGemm4Args, "ra_linear4_grad_args": _lib.RaLinear4GradArgs, "ra_grad": _lib.RaGrad,
               "ra_adamw_tensor": _lib.RaAdamwTensor, "ra_adamw_args": _lib.RaAdamwArgs}
    lines, want = [], []
    for name, cls in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for field, *_ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field))
            want.append(getattr(cls, field).offset)
    for c in ("RA_Q4_E4M3", "RA_Q4_E8M0", "RA_F32", "RA_BF16"):
        lines.append('printf("%%d\\n", (int)%s);' % c)
        want.append(getattr(_lib, c))
    src = tmp_path / "layout4.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"refadapt.h\"\nint main(void) {\n%s\nreturn 0;\n}\n"
                   % "\n".join(lines))
    exe = tmp_path / "layout4"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == want


def test_sizes(lib):
    size = lib.refadapt_quant4_scales_size
    for rows, K, fmt, want in ((1, 64, 0, 512), (128, 64, 0, 512), (129, 64, 0, 1024), (1, 65, 0, 1024), (128, 128, 1, 512),
                               (256, 192, 1, 2048), (0, 64, 0, 0), (5, 0, 0, 0), (-1, 64, 0, 0), (1, 64, 2, 0),
                               (2147483647, 64, 0, 2 ** 24 * 512)):
        assert size(rows, K, fmt) == want, (rows, K, fmt)
    assert lib.refadapt_linear4_backward_workspace_size(0, 1, 64, 64) == 0
    assert lib.refadapt_linear4_backward_workspace_size(1, 0, 64, 64) >= 16
    assert lib.refadapt_linear4_backward_workspace_size(2, 100, 64, 128) > 200 * 64 + 128 * 32 + 64 * 128
    assert lib.refadapt_grad_norm_workspace_size() > 16


def quant(both=False):
    from paper_2609_32415_gb300 import _lib
    a = _lib.RaQuant4Args()
    a.B, a.C, a.n_seg, a.format = 1, 128, 1, 0
    s = a.seg[0]
    s.x, s.x_stride_s, s.x_stride_r, s.rows = 0x100000, 128 * 40, 128, 40
    s.codes, s.codes_stride_s, s.codes_stride_r, s.scales = 0x200000, 64 * 40, 64, 0x300000
    if both:
        s.codes_t, s.codes_t_stride, s.scales_t = 0x400000, 32, 0x500000
    return a


def test_quant4_refuses(lib):
    call = lambda a: lib.refadapt_quant4(ctypes.byref(a), None)  # noqa: E731
    refused(lib, lib.refadapt_quant4(None, None), b"args is NULL")
    for field, value, text in (("B", 0, b"B >= 1"), ("C", 12, b"multiple of 8"), ("C", 72, b"multiple of 64"),
                               ("n_seg", 4, b"n_seg"), ("format", 2, b"format")):
        a = quant()
        setattr(a, field, value)
        refused(lib, call(a), text)
    for field, value, text in (("rows", -1, b"rows"), ("rows", 1 << 30, b"2^30"), ("x", 0x100008, b"16-byte"), ("x", None, b"x must"),
                               ("x_stride_r", 120, b">= C"), ("x_stride_r", 132, b"multiples of 8"), ("codes", None, b"go with"),
                               ("scales", None, b"go with"), ("scales", 0x300008, b"16-byte"), ("codes", 0x200004, b"16-byte"),
                               ("codes_stride_r", 72, b"16 bytes"), ("codes_stride_r", 48, b"C / 2"), ("gated", 1, b"gated"),
                               ("exponent", 65, b"exponent"), ("codes", 0x100000, b"overlaps"),
                               ("scales", 0x200000 + 64, b"overlaps")):
        a = quant()
        setattr(a.seg[0], field, value)
        refused(lib, call(a), text)
    a = quant()
    a.format, a.seg[0].exponent = 1, 1
    refused(lib, call(a), b"0 for RA_Q4_E8M0")
    for field, value, text in (("scales_t", None, b"go with"), ("codes_t_stride", 16, b"holds all rows"),
                               ("codes_t_stride", 40, b"16 bytes"), ("codes_t", 0x300000, b"overlaps")):
        a = quant(both=True)
        setattr(a.seg[0], field, value)
        refused(lib, call(a), text)
    a = quant(both=True)
    a.seg[0].gated, a.mode = 1, 0x600000
    refused(lib, call(a), b"codes_t")
    a = quant()
    a.seg[0].codes = a.seg[0].scales = None
    refused(lib, call(a), b"no outputs")


def gemm(epilogue=0):
    from paper_2609_32415_gb300 import _lib
    a = _lib.RaGemm4Args()
    a.B, a.N, a.K, a.n_seg, a.epilogue = 1, 768, 128, 1, epilogue
    s, q = a.seg[0].lin, a.seg[0]
    s.a, s.a_stride_s, s.a_stride_r, s.rows, s.w = 0x100000, 64 * 40, 64, 40, 0x200000
    q.a_scales, q.w_scales = 0x300000, 0x400000
    s.out, s.out_stride_s, s.out_stride_r = 0x500000, 768 * 40, 768
    if epilogue == 2:
        s.resid, s.resid_stride_s, s.resid_stride_r, s.gate = 0x700000, 768 * 40, 768, 0x900000
    if epilogue == 3:
        a.H, a.d, a.rope, a.rope_len, a.norm_eps = 4, 64, 0xa00000, 64, 1e-6
        s.q_norm = s.k_norm = 0xb00000
        s.q_out, s.k_out, s.v_out = (_lib.RaSeg(p, 256 * 40, 64 * 40, 64, 40, 0) for p in (0xc00000, 0xd00000, 0xe00000))
    return a


def test_gemm4_refuses(lib):
    call = lambda a: lib.refadapt_gemm4(ctypes.byref(a), None)  # noqa: E731
    refused(lib, lib.refadapt_gemm4(None, None), b"args is NULL")
    for field, value, text in (("B", 0, b"B >= 1"), ("N", 96, b"multiples of 64"), ("K", 96, b"multiples of 64"), ("K", 0, b"positive"),
                               ("n_seg", 0, b"n_seg"), ("epilogue", 4, b"epilogue"), ("format", 2, b"format"),
                               ("tile_mode", 3, b"tile_mode")):
        a = gemm()
        setattr(a, field, value)
        refused(lib, call(a), text)
    for field, value, text in (("rows", -1, b"rows"), ("gated", 1, b"gated"), ("a", 0x100008, b"16-byte"), ("a", None, b"16-byte"),
                               ("w", 0x200004, b"16-byte"), ("a_stride_r", 48, b"K / 2"), ("a_stride_r", 72, b"16 bytes"),
                               ("bias", 0x4, b"bias"), ("out", None, b"out must"), ("out_stride_r", 760, b">= N"),
                               ("out", 0x100000, b"overlaps"), ("out", 0x200000 + 64 * 768 - 32, b"overlaps"),
                               ("out", 0x400000, b"overlaps")):
        a = gemm()
        setattr(a.seg[0].lin, field, value)
        refused(lib, call(a), text)
    for field, value, text in (("a_scales", None, b"scales"), ("w_scales", 0x400008, b"16-byte"), ("a_exponent", 65, b"exponents"),
                               ("w_exponent", -65, b"exponents")):
        a = gemm()
        setattr(a.seg[0], field, value)
        refused(lib, call(a), text)
    a = gemm()
    a.format, a.seg[0].w_exponent = 1, 2
    refused(lib, call(a), b"0 for RA_Q4_E8M0")
    a = gemm()
    a.B, a.seg[0].lin.out_stride_s = 2, 0
    refused(lib, call(a), b"positive")
    for field, value, text in (("resid", None, b"resid"), ("gate", 0x900004, b"16-byte"), ("resid", 0x500000 + 768 * 2, b"overlaps")):
        a = gemm(2)
        setattr(a.seg[0].lin, field, value)
        refused(lib, call(a), text)
    for change, text in ((dict(d=32), b"QKV needs d"), (dict(H=3), b"N = 3 H d"), (dict(rope=None), b"rope"),
                         (dict(rope_len=39), b"outside")):
        a = gemm(3)
        for k, v in change.items():
            setattr(a, k, v)
        refused(lib, call(a), text)
    a = gemm(3)
    a.seg[0].lin.k_out.ptr = a.seg[0].lin.q_out.ptr
    refused(lib, call(a), b"overlaps")
    a = gemm(3)
    a.seg[0].lin.v_out.stride_n = 0
    refused(lib, call(a), b"strides")
    a = gemm()  # segments that share an output
    a.n_seg = 2
    ctypes.memmove(ctypes.byref(a.seg[1]), ctypes.byref(a.seg[0]), ctypes.sizeof(a.seg[0]))
    refused(lib, call(a), b"overlaps")


def grad():
    from paper_2609_32415_gb300 import _lib
    a = _lib.RaLinear4GradArgs()
    a.B, a.rows, a.K, a.N = 2, 20, 128, 192
    a.dy, a.dy_stride_s, a.dy_stride_r = 0x100000, 192 * 20, 192
    a.x, a.x_stride_s, a.x_stride_r, a.w = 0x200000, 128 * 20, 128, 0x300000
    a.dx, a.dx_stride_s, a.dx_stride_r, a.dw = 0x400000, 128 * 20, 128, 0x500000
    a.workspace, a.workspace_bytes = 0x1000000, 1 << 20
    return a


def test_linear4_backward_refuses(lib):
    call = lambda a: lib.refadapt_linear4_backward(ctypes.byref(a), None)  # noqa: E731
    refused(lib, lib.refadapt_linear4_backward(None, None), b"args is NULL")
    for field, value, text in (("B", 0, b"B >= 1"), ("rows", -1, b"rows"), ("rows", 1 << 29, b"2^30"), ("K", 96, b"multiples of 64"),
                               ("N", 0, b"positive"), ("dy", None, b"dy"), ("dy", 0x100002, b"16-byte"), ("x", None, b"x (with dw)"),
                               ("w", None, b"w and dx"), ("dw", 0x500004, b"dw"), ("dx", 0x400008, b"16-byte"),
                               ("x_stride_r", 64, b"at least a row"), ("dx_stride_s", 128 * 24, b"follow"),
                               ("dx_stride_s", 0, b"follow"), ("workspace", None, b"workspace"), ("workspace", 0x1000008, b"workspace"),
                               ("workspace_bytes", 1000, b"bytes"), ("workspace", 0x500000, b"overlaps"), ("dw", 0x300000, b"overlaps"),
                               ("dx", 0x200000, b"overlaps"), ("dx", 0x100000, b"overlaps")):
        a = grad()
        setattr(a, field, value)
        refused(lib, call(a), text)
    a = grad()
    a.dx = a.dw = None
    refused(lib, call(a), b"neither")


def test_grad_norm_refuses(lib):
    from paper_2609_32415_gb300 import _lib
    size = lib.refadapt_grad_norm_workspace_size()
    t = (_lib.RaGrad * 2)(_lib.RaGrad(0x100000, 100, 0, 0), _lib.RaGrad(0x200000, 0, 1, 0))
    good = dict(t=t, n=2, most=1.0, out=0x300000, ws=0x400000, size=size)

    def call(**kw):
        a = dict(good, **kw)
        return lib.refadapt_grad_norm(a["t"], a["n"], a["most"], a["out"], a["ws"], a["size"], None)

    for kw, text in ((dict(n=-1), b"n_tensors"), (dict(t=None), b"array"), (dict(most=0.0), b"max_norm"),
                     (dict(most=float("nan")), b"max_norm"), (dict(out=None), b"out"), (dict(ws=None), b"workspace"),
                     (dict(ws=0x400004), b"workspace"), (dict(size=size - 1), b"bytes"), (dict(out=0x400010), b"overlap"),
                     (dict(out=0x100004), b"overlaps"), (dict(ws=0x100040), b"overlaps")):
        refused(lib, call(**kw), text)
    for field, value in (("n", -1), ("n", (1 << 42) + 1), ("type", 2), ("g", None), ("g", 0x100002)):
        u = (_lib.RaGrad * 1)(_lib.RaGrad(0x100000, 100, 0, 0))
        setattr(u[0], field, value)
        refused(lib, call(t=u, n=1), b"tensor 0")


def test_adamw_refuses(lib):
    from paper_2609_32415_gb300 import _lib

    def tensor(base, n=100):
        return _lib.RaAdamwTensor(base, base + 0x1000, base + 0x2000, base + 0x3000, base + 0x4000, base + 0x5000, base + 0x6000,
                                  n, 0, 0)

    def args(*ts, bits=32, **kw):
        arr = (_lib.RaAdamwTensor * max(1, len(ts)))(*ts)
        a = _lib.RaAdamwArgs(arr, len(ts), bits, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, 0)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    call = lambda a: lib.refadapt_adamw(ctypes.byref(a), None)  # noqa: E731
    refused(lib, lib.refadapt_adamw(None, None), b"args is NULL")
    for kw, text in ((dict(bits=16), b"bits"), (dict(n_tensors=-1), b"n_tensors"), (dict(beta1=1.0), b"betas"),
                     (dict(beta2=-0.1), b"betas"), (dict(beta1=float("nan")), b"betas"), (dict(eps=0.0), b"eps"),
                     (dict(decay=-1.0), b"decay"), (dict(lr=-1e-3), b"lr"), (dict(lr=float("inf")), b"lr"), (dict(step=0), b"step"),
                     (dict(step=1 << 31), b"step")):
        refused(lib, call(args(tensor(0x100000), **kw)), text)
    for field, value in (("p", None), ("g", None), ("m", None), ("v", None), ("p", 0x100002), ("w", 0x100001), ("n", -1),
                         ("g_type", 2), ("m", 0x102002)):
        t = tensor(0x100000)
        setattr(t, field, value)
        refused(lib, call(args(t)), b"tensor 0")
    for field in ("m_scale", "v_scale"):
        t = tensor(0x100000)
        setattr(t, field, None)
        refused(lib, call(args(t, bits=8)), b"m_scale")
    # one tensor twice; a gradient that is another's weight; moments that meet; a scale inside a weight
    refused(lib, call(args(tensor(0x100000), tensor(0x100000))), b"overlaps")
    for field, value in (("g", 0x100000), ("m", 0x10018c), ("w", 0x10218c), ("v", 0x106000)):
        t = tensor(0x200000)
        setattr(t, field, value)
        refused(lib, call(args(tensor(0x100000), t)), b"overlaps")
    refused(lib, call(args(tensor(0x100000), grad_scale=0x100010)), b"overlaps")
    t = tensor(0x100000)
    t.v_scale = t.m_scale + 3  # four bytes each
    refused(lib, call(args(t, bits=8)), b"overlaps")


def test_binding_checks_tensors():
    """Wrong tensors are refused by the binding before the library sees them (CPU tensors among them)."""
    import torch
    from paper_2609_32415_gb300 import api
    x = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x: expected"):
        api.refadapt_quant4([{"x": x, "codes": x, "scales": x}], 64, 0)
    with pytest.raises(ValueError, match="a: expected"):
        api.refadapt_gemm4([{"a": torch.zeros((1, 4, 32), dtype=torch.uint8)}], 64, 64, 0, 0)
    with pytest.raises(KeyError):
        api.refadapt_gemm4([{}], 64, 64, 0, 0)
    with pytest.raises(ValueError, match="dy"):
        api.refadapt_linear4_backward(x, x, torch.zeros((64, 64), dtype=torch.bfloat16), x)
    with pytest.raises(ValueError, match="grads"):
        api.refadapt_grad_norm([torch.zeros(3)], 1.0, torch.zeros(2), torch.zeros(1))
    with pytest.raises(ValueError, match="p: expected"):
        api.refadapt_adamw([{"p": torch.zeros(3)}], 1e-3, 1)
    with pytest.raises(TypeError):
        api.refadapt_quant4([], 64, 0)
    with pytest.raises(ValueError, match="32 or 8"):
        api.adamw_moments(torch.zeros(3), 4)
    with pytest.raises(ValueError, match="N, K"):
        api.weight4(torch.zeros(3))
