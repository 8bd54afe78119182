"""RefAdapt-DiT hot path on GB300 (sm_103a).

librefadapt.so (C ABI, include/refadapt.h) holds every kernel: joint attention
with the reference mass on tcgen05 tensor cores, the target-Q change
reduction, the first-crossing gate and the reference-cache update, and the
layers of the DiT block around the attention (tcgen05 GEMM with fused
epilogues, modulated LayerNorm, RoPE table; for gated blocks also the gated
feed-forward, the norms around a branch and rotary positions with several axes,
with their backward passes; linear layers in microscaled 4 bits, forward and
backward; the optimiser's step). This package is its thin binding (``api``),
Algorithm 1's host loop over the attention (``executor``), over a stack of DiT
blocks (``dit``) and of gated DiT blocks (``gated_dit``), the gated layers and the
4-bit ones as autograd functions with an optimiser (``training``), and the seeded synthetic input generator
(``synth``). Calls fail loudly when
the library has not been built; nothing falls back to the CPU.
"""
from . import api, synth  # noqa: F401
from ._lib import (RA_MODE_BOUNDARY, RA_MODE_COMPUTE, RA_MODE_FULL, RA_MODE_REUSE, RA_Q4_E4M3,  # noqa: F401
                   RA_Q4_E8M0, RefAdaptError)
from .dit import DiTExecutor  # noqa: F401
from .executor import Executor, roles_from_joint  # noqa: F401
from .gated_dit import GatedDiTExecutor  # noqa: F401

__version__ = "0.1.0"
