"""Calls of the 4-bit products and of the optimiser that the host refuses: numbers that are none in fp32, exponents
whose product is none, outputs that meet other tensors anywhere (no GPU needed)."""
import ctypes

import pytest

from test_abi_layers_cpu import refused
from test_abi_linear4_cpu import gemm, grad, lib, quant  # noqa: F401


@pytest.mark.parametrize("field, value", [("eps", 1e-39), ("eps", 1e-46), ("eps", 5e-324), ("eps", -1.0), ("eps", 1e39),
                                          ("lr", 1e39), ("decay", 1e39), ("eps", float("nan"))])
def test_adamw_refuses_rates_that_fp32_does_not_have(lib, field, value):  # noqa: F811
    from paper_2609_32415_gb300 import _lib
    t = (_lib.RaAdamwTensor * 1)(_lib.RaAdamwTensor(*(0x100000 + 0x1000 * i for i in range(7)), 100, 0, 0))
    a = _lib.RaAdamwArgs(t, 1, 32, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, 0)
    setattr(a, field, value)
    refused(lib, lib.refadapt_adamw(ctypes.byref(a), None), b"finite in fp32")


def test_gemm4_refuses_outputs_that_meet_other_tensors_anywhere(lib):  # noqa: F811
    """Other heads than the first, later rows, the rotary table, the norm weights, the modes; heads, rows and samples
    of one output that meet each other."""
    call = lambda a: lib.refadapt_gemm4(ctypes.byref(a), None)  # noqa: E731
    a = gemm(3)  # 4 heads of 40 rows of 64: 20,480 bytes from 0xc00000, 0xd00000 and 0xe00000 on
    for part, field, value in (("lin", "q_norm", 0xc00000 + 20224), ("lin", "k_norm", 0xd00000 + 5120 * 3),
                               ("lin", "bias", 0xe00000 + 20480 - 16), ("lin", "w", 0xc00000 - 768 * 64 + 16),
                               ("lin", "a", 0xd00000 + 20480 - 16), (None, "a_scales", 0xe00000 + 10240),
                               (None, "w_scales", 0xe00000 + 20480 - 512)):
        a = gemm(3)
        setattr(a.seg[0].lin if part else a.seg[0], field, value)
        refused(lib, call(a), b"overlaps")
    for field, value in (("rope", 0xc00000 + 20480 - 16), ("mode", 0xd00000 + 40), ("err_word", 0xe00000 + 20476)):
        a = gemm(3)
        setattr(a, field, value)
        refused(lib, call(a), b"overlaps")
    for shift in (16, 5120, 20480 - 128):
        a = gemm(3)
        a.seg[0].lin.k_out.ptr = 0xc00000 + shift
        refused(lib, call(a), b"overlaps")
    for stride_h, stride_n in ((8, 64), (64, 64), (32, 256), (64 * 39, 64), (64, 128)):
        a = gemm(3)
        a.seg[0].lin.v_out.stride_h, a.seg[0].lin.v_out.stride_n = stride_h, stride_n
        refused(lib, call(a), b"itself")
    # side by side in one buffer of rows of 768, and k eight columns too early
    a = gemm(3)
    for z, at in (("q_out", 0), ("k_out", 512 - 16), ("v_out", 1024)):
        o = getattr(a.seg[0].lin, z)
        o.ptr, o.stride_b, o.stride_h, o.stride_n = 0xc00000 + at, 768 * 40, 64, 768
    refused(lib, call(a), b"overlaps")
    a = gemm()  # rows in a wider buffer that the weight's end reaches into
    a.seg[0].lin.out_stride_r, a.seg[0].lin.out_stride_s = 1024, 1024 * 40
    a.seg[0].lin.w = 0x500000 + 2048 * 39 + 1024
    refused(lib, call(a), b"overlaps")
    a = gemm()
    a.B, a.seg[0].lin.out_stride_s = 2, 768 * 39
    refused(lib, call(a), b"itself")


def test_gemm4_refuses_exponents_that_pass_fp32_together(lib):  # noqa: F811
    a = gemm()
    a.seg[0].a_exponent = a.seg[0].w_exponent = 64
    refused(lib, lib.refadapt_gemm4(ctypes.byref(a), None), b"together at most 127")


def test_quant4_and_gradients_refuse_outputs_that_meet_rows_of_wider_buffers(lib):  # noqa: F811
    call = lambda a: lib.refadapt_quant4(ctypes.byref(a), None)  # noqa: E731
    for field, value in (("codes", 0x100000 + 512 * 3 + 240), ("scales", 0x100000 + 512 * 39 + 16), ("codes_t", 0x100000 + 512 * 20),
                         ("scales_t", 0x100000 - 512 + 16)):
        a = quant(both=True)  # rows of 256 bytes, 512 apart
        a.seg[0].x_stride_r, a.seg[0].x_stride_s = 256, 256 * 40
        setattr(a.seg[0], field, value)
        refused(lib, call(a), b"overlaps")
    a = quant()  # the second sample begins in the first one's last row
    a.B, a.seg[0].codes_stride_s = 2, 64 * 40 - 16
    refused(lib, call(a), b"itself")
    a = quant()
    a.seg[0].gated, a.mode = 1, 0x200000 + 64 * 39
    refused(lib, call(a), b"overlaps")

    call = lambda a: lib.refadapt_linear4_backward(ctypes.byref(a), None)  # noqa: E731
    for field, value in (("dx", 0x100000 + 512 * 30 + 128), ("dw", 0x100000 + 512 * 39 + 368), ("workspace", 0x100000 + 512 * 39),
                         ("err_word", 0x500000 + 128 * 192 * 2 - 4)):
        a = grad()  # dy: rows of 384 bytes, 512 apart
        a.dy_stride_r, a.dy_stride_s = 256, 256 * 20
        setattr(a, field, value)
        refused(lib, call(a), b"overlaps")
