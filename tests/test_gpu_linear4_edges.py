"""4-bit products at the ends of what they take: row tiles that end early one after another, values and
exponents at the ends of their ranges. Bounds as in test_gpu_linear4 (exact 4-bit operands, K 2^-23 sum |a w|
for the fp32 sums, half a bf16 step, 2^-20 of what enters an epilogue)."""
import numpy as np
import pytest
import torch

from test_gpu_linear4 import (BF, E4M3, E8M0, F32, GELU, QKV, RESID, STORE, api, bf, f64, f64_32, gelu64, operands, values_of,
                              within)

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


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("tile_mode, rows", [(0, 1), (1, 2), (2, 2)])
def test_gelu_at_its_ends(cuda_ok, fmt, tile_mode, rows):
    """x from the bias, the products being zero: what is far below zero gives nothing, at minus infinity as well, NaN
    and infinity stay where they are, in the kernel of one row and in the tiles alike. x (1 + e^z)^-1 is below 8 2^-60
    from -7.5 on, so 2^-56 is allowed there; above, three roundings of an exponent up to 60 are
    within 2^-16 of the value."""
    a, K = api(), 128
    inf = float("inf")
    x = [-inf, 1.0, -3e38, -1e30, inf, -1e18, float("nan"), -2.0, -1e6, -1000.0, -100.0, -20.0, -10.0, -8.0, -7.6, -7.5, -7.4, -7.0,
         -6.0, -5.0, -4.0, -3.0, -1.0, -1e-3, 0.0, 1e-30, 1e-3, 0.5, 3.0, 7.0, 20.0, 1e6, 1e18, 3e38, float("nan"), -1e20]
    x = np.array(x + [-0.25 * i for i in range(64 - len(x))])
    N = 64
    seg, _, _ = operands(1, rows, N, K, fmt, torch.Generator().manual_seed(1))
    seg["a"].zero_()
    seg["bias"] = torch.tensor(x, dtype=torch.float32, device="cuda")
    x = seg["bias"].double().cpu().numpy()
    seg["out"] = torch.zeros((1, rows, N), dtype=torch.bfloat16, device="cuda")
    a.refadapt_gemm4([seg], N, K, GELU, fmt, tile_mode=tile_mode)
    with np.errstate(all="ignore"):
        ref = np.where(x == -inf, 0.0, x / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3))))
    got = seg["out"].double().cpu().numpy()[0]
    plain = np.isfinite(x) | (x == -inf)
    for r in range(rows):
        assert np.isnan(got[r][np.isnan(x)]).all() and (got[r][x == inf] == inf).all()
        assert np.isfinite(got[r][plain]).all()
        assert (np.abs(got[r][plain] - ref[plain]) <= (BF + 2.0 ** -15) * np.abs(ref[plain]) + 2.0 ** -56).all()


@pytest.mark.parametrize("tile_mode, rows", [(0, 1), (0, 40), (2, 300)])
@pytest.mark.parametrize("exps", [(64, 63), (63, 64), (-64, -63), (-64, -64), (64, -64)])
def test_exponents_at_their_ends(cuda_ok, tile_mode, rows, exps):
    """2^127 and 2^-128 are numbers; half a step of bf16's smallest ones is 2^-134 (and fp32's 2^-150)."""
    a, N, K = api(), 128, 192
    g = torch.Generator().manual_seed(rows)
    seg, _, _ = operands(1, rows, N, K, E4M3, g, 0, -6)
    seg.update(a_exponent=exps[0], w_exponent=exps[1])
    if sum(exps) > 100:  # scales of 2^-9 on both sides: values of one over K times 2^127 at most
        seg["a_scales"].clamp_(max=1)
        seg["w_scales"].clamp_(max=1)
    p = values_of(seg["a"][0], seg["a_scales"][0], E4M3, exps[0])
    q = values_of(seg["w"], seg["w_scales"], E4M3, exps[1])
    ref = p @ q.T
    assert np.abs(ref).max() < 2.0 ** 126
    seg["out"] = torch.zeros((1, rows, N), dtype=torch.bfloat16, device="cuda")
    a.refadapt_gemm4([seg], N, K, STORE, E4M3, tile_mode=tile_mode)
    within(seg["out"][0], ref, BF * np.abs(ref) + K * 2.0 ** -23 * (np.abs(p) @ np.abs(q).T) + 2.0 ** -133.9)


@pytest.mark.parametrize("d", [64, 128])
def test_qkv_side_by_side(cuda_ok, d):
    """q, k and v as parts of one buffer of rows, and in slots of a longer cache: what separate tensors hold, and
    nothing beside them is touched."""
    a, g = api(), torch.Generator().manual_seed(d)
    B, rows, K, H = 2, 70, 128, 512 // d
    N = 3 * H * d
    norm = torch.linspace(0.5, 1.5, d, device="cuda")
    seg, _, _ = operands(B, rows, N, K, E8M0, g)

    def run(q, k, v):
        a.refadapt_gemm4([{**seg, "q": q, "k": k, "v": v, "q_norm": norm, "k_norm": norm, "pos_offset": 3}], N, K, QKV, E8M0,
                         rope=a.rope_table(rows + 3, d), H=H, d=d)
        return q, k, v

    def empty(*s):
        return torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")

    want = run(*(empty(B, H, rows, d) for _ in range(3)))
    whole = empty(B, rows + 1, 3, H, d)
    side = run(*(whole[:, :rows, i].transpose(1, 2) for i in range(3)))
    cache = empty(B, 2, H, rows + 40, d)
    slots = run(empty(B, H, rows, d), cache[:, 0, :, 11:11 + rows], cache[:, 1, :, 11:11 + rows])
    two = empty(B, H, 2 * rows, d)  # q and k take turns along the rows of one tensor
    turns = run(two[:, :, ::2], two[:, :, 1::2], empty(B, H, rows, d))
    for got in (side, slots, turns):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert bool((whole[:, rows] == 7.0).all())
    assert bool((cache[:, :, :, :11] == 7.0).all()) and bool((cache[:, :, :, 11 + rows:] == 7.0).all())
