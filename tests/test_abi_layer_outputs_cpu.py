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
