"""Calls of the 4-bit products and of the optimiser that the host refuses: numbers that are none in fp32, exponents
whose product is none, outputs that meet other tensors anywhere (no GPU needed)."""
import ctypes

import pytest

from test_abi_layers_cpu import refused
from test_abi_linear4_cpu import lib  # noqa: F401


@pytest.mark.parametrize("field, value", [("eps", 1e-39), ("eps", 1e-46), ("eps", 5e-324), ("eps", -1.0), ("eps", 1e39),
                                          ("lr", 1e39), ("decay", 1e39), ("eps", float("nan"))])
def test_adamw_refuses_rates_that_fp32_does_not_have(lib, field, value):  # noqa: F811
    from paper_2609_32415_gb300 import _lib
    t = (_lib.RaAdamwTensor * 1)(_lib.RaAdamwTensor(*(0x100000 + 0x1000 * i for i in range(7)), 100, 0, 0))
    a = _lib.RaAdamwArgs(t, 1, 32, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, 0)
    setattr(a, field, value)
    refused(lib, lib.refadapt_adamw(ctypes.byref(a), None), b"finite in fp32")
