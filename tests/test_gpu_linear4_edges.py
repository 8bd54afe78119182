"""4-bit products at the ends of what they take: row tiles that end early one after another, values and
exponents at the ends of their ranges. Bounds as in test_gpu_linear4 (exact 4-bit operands, K 2^-23 sum |a w|
for the fp32 sums, half a bf16 step, 2^-20 of what enters an epilogue)."""
import numpy as np
import pytest
import torch

from oracle import lowbit
from test_gpu_linear4 import (BF, E4M3, E8M0, F32, GELU, QKV, RESID, STORE, api, bf, f64, f64_32, gelu64, operands, quantised,
                              values_of, within)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("tile_mode", [1, 2])
@pytest.mark.parametrize("epilogue, rows, d", [(STORE, 17, 0), (GELU, 33, 0), (RESID, 1, 0), (RESID, 97, 0), (QKV, 17, 64),
                                               (QKV, 31, 128)])
def test_partial_row_tiles_one_after_another(cuda_ok, fmt, tile_mode, epilogue, rows, d):
    """Samples of few rows, each a row tile that ends early, several tiles of columns with biases (and gates) of
    their own: a warp goes on to the next tile's vectors although most of its lanes have no row to store."""
    a, g = api(), torch.Generator().manual_seed(rows + epilogue)
    B, K, N = 200, 64, 768 if epilogue == QKV else 832
    seg, y, acc = operands(B, rows, N, K, fmt, g)
    seg["bias"] = torch.randn(N, generator=g).cuda()
    x = y + f64_32(seg["bias"])
    e = acc + F32 * (np.abs(x) + np.abs(y))
    kw, want = {}, []
    if epilogue == QKV:
        H = N // 3 // d
        rope = a.rope_table(rows, d)
        norm = {z: (1 + 0.2 * torch.randn(d, generator=g)).cuda() for z in ("q_norm", "k_norm")}
        for z in "qkv":
            seg[z] = torch.full((B, H, rows, d), 7.0, dtype=torch.bfloat16, device="cuda")
        seg.update(norm, pos_offset=0)
        kw = dict(rope=rope, H=H, d=d)
        x, e = (t.reshape(B, rows, 3, H, d).transpose(2, 0, 3, 1, 4) for t in (x, e))
        c, s = (f64_32(rope)[..., i] for i in (0, 1))
        for i, z in enumerate("qkv"):
            if z == "v":
                want.append((seg[z], x[i], BF * np.abs(x[i]) + e[i]))
                continue
            rms, w = np.sqrt((x[i] ** 2).mean(-1, keepdims=True) + 1e-6), f64_32(norm[z + "_norm"])
            n = x[i] / rms * w
            ref = np.empty_like(n)
            ref[..., 0::2] = n[..., 0::2] * c - n[..., 1::2] * s
            ref[..., 1::2] = n[..., 0::2] * s + n[..., 1::2] * c
            top = np.abs(n).max(-1, keepdims=True)
            want.append((seg[z], ref, BF * np.abs(ref) + 2 * e[i].max(-1, keepdims=True) / rms * (np.abs(w).max() + top) +
                         4 * F32 * top))
    else:
        seg["out"] = torch.full((B, rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
        if epilogue == GELU:
            ref, tol = gelu64(x), 1.2 * e + 16 * F32 * np.abs(x)
        elif epilogue == RESID:
            seg.update(gate=torch.randn((B, N), generator=g).cuda(), resid=bf((B, rows, N), g))
            gate = f64_32(seg["gate"])[:, None]
            ref = f64(seg["resid"]) + gate * x
            tol = np.abs(gate) * e + F32 * np.abs(ref)
        else:
            ref, tol = x, e
        want.append((seg["out"], ref, tol + BF * np.abs(ref)))
    a.refadapt_gemm4([seg], N, K, epilogue, fmt, tile_mode=tile_mode, **kw)
    for got, ref, tol in want:
        within(got, ref, tol + 1e-30)
