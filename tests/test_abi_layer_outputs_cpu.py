"""Outputs of the gated block's layers that would race with an input or with one
another are refused before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest

from test_abi_layers_cpu import refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_32415_gb300 import _lib, build
    build.build()
    return _lib.load()


def rope_args(tensors, B=2, n=4, d=64, heads=3):
    """tensors: (x, out) pairs of (address, sample, head, row stride)."""
    from paper_2609_32415_gb300 import _lib
    a = _lib.RaRopeArgs()
    a.B, a.n, a.d, a.n_axes, a.base, a.n_tensors, a.pos = B, n, d, 1, 1e4, len(tensors), 0x40000
    a.axis_dim[0] = d
    for i, (x, out) in enumerate(tensors):
        a.t[i].heads = heads
        a.t[i].x = _lib.RaSeg(*x, n, 0)
        a.t[i].out = _lib.RaSeg(*out, n, 0)
    return a


HEAD_MAJOR, TOKEN_MAJOR = (768, 256, 64), (768, 64, 192)


def test_rope_in_place_needs_the_same_strides(lib):
    a = rope_args([((0x10000, *HEAD_MAJOR), (0x10000, *TOKEN_MAJOR))])
    refused(lib, lib.refadapt_rope_axes(ctypes.byref(a), None), b"in place")


@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("stride", [0, 56])
def test_rope_output_with_rows_on_one_another(lib, axis, stride):
    strides = list(HEAD_MAJOR)
    strides[axis] = stride
    a = rope_args([((0x10000, *HEAD_MAJOR), (0x20000, *strides))])
    refused(lib, lib.refadapt_rope_axes(ctypes.byref(a), None), b"one another")


def test_rope_tensors_that_share_an_output(lib):
    x, y, z = (0x10000, *HEAD_MAJOR), (0x20000, *HEAD_MAJOR), (0x30000, *HEAD_MAJOR)
    for pairs in ([(x, z), (y, z)], [(x, y), (y, z)], [(y, z), (x, y)], [(x, x), (x, x)]):
        a = rope_args(pairs)
        refused(lib, lib.refadapt_rope_axes(ctypes.byref(a), None), b"the other's")


# ------------------------------------------------------------------ gated feed-forward
ROWS, C, F = 4, 64, 128


def glu_args(places):
    """Segments of x, w_gate, w_up, out, pre_gate, pre_up at these addresses, rows dense."""
    from paper_2609_32415_gb300 import _lib
    a = _lib.RaGluArgs()
    a.B, a.F, a.C, a.act, a.n_seg = 1, F, C, 0, len(places)
    for s, at in zip(a.seg, places):
        s.rows = ROWS
        for name, ptr in zip(("x", "w_gate", "w_up", "out", "pre_gate", "pre_up"), at):
            setattr(s, name, ptr)
        for name, width in (("x", C), ("out", F), ("pre_gate", F), ("pre_up", F)):
            setattr(s, name + "_stride_s", ROWS * width)
            setattr(s, name + "_stride_r", width)
    return a


@pytest.mark.parametrize("which,at", [
    (3, (1, 0)), (3, (1, 3)), (5, (1, 4)),    # out = the other segment's x, out; pre_up = its pre_gate
    (3, (0, 1)), (4, (1, 2)),                 # a weight of its own, of the other segment
    (4, (0, 5)),                              # pre_gate = pre_up
])
@pytest.mark.parametrize("offset", [0, 16])
def test_glu_outputs_that_overlap(lib, which, at, offset):
    places = [[0x100000 * (6 * s + i + 1) for i in range(6)] for s in range(2)]
    places[0][which] = places[at[0]][at[1]] + offset
    refused(lib, lib.refadapt_glu(ctypes.byref(glu_args(places)), None), b"overlap")


@pytest.mark.parametrize("out", ["dx", "dw_gate", "dw_up", "dw_down", "workspace"])
@pytest.mark.parametrize("other", ["dy", "x", "pre_gate", "pre_up", "hidden", "w_gate", "w_up", "w_down", "dx", "dw_gate",
                                   "dw_up", "dw_down", "workspace"])
def test_glu_gradients_that_overlap(lib, out, other):
    from paper_2609_32415_gb300 import _lib
    if out == other:
        return
    b = _lib.RaGluGradArgs()
    b.B, b.rows, b.C, b.F, b.O, b.act = 1, ROWS, C, F, C, 0
    names = ("dy", "x", "pre_gate", "pre_up", "hidden", "w_gate", "w_up", "w_down", "dx", "dw_gate", "dw_up", "dw_down",
             "workspace")
    for i, name in enumerate(names):
        setattr(b, name, 0x100000 * (i + 1))
    for name, width in (("dy", C), ("x", C), ("pre_gate", F), ("pre_up", F), ("hidden", F), ("dx", C)):
        setattr(b, name + "_stride_s", ROWS * width)
        setattr(b, name + "_stride_r", width)
    b.workspace_bytes = lib.refadapt_glu_backward_workspace_size(1, ROWS, C, F, C)
    for offset in (0, 16):
        setattr(b, out, getattr(b, other) + offset)
        refused(lib, lib.refadapt_glu_backward(ctypes.byref(b), None), b"overlap")
