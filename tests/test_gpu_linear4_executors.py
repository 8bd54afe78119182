"""The executors' QKV products with 4-bit weights, on the rows that entered them: positions, cache slots and modes
as the block defines them, not as the call was made. Bounds as in test_gpu_linear4.test_qkv."""
import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import dit as oracle_dit
from oracle import layers, lowbit
from test_gpu_gated_block import AXES, make
from test_gpu_linear4 import BF, F32, within
from test_gpu_linear4_layers import mlp_weights, quantise_weights

pytestmark = pytest.mark.gpu
REUSE, BOUNDARY, COMPUTE, FULL = 0, 1, 2, 3
STREAM_OF = {"text": "text", "ref": "image", "tgt": "image"}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name, exponent", [("e4m3", 0), ("e4m3", -3), ("e8m0", 0)])
def test_qkv_of_every_role_and_mode(cuda_ok, monkeypatch, gated, name, exponent):
    from paper_2609_32415_gb300 import DiTExecutor, GatedDiTExecutor, dit
    fmt = {"e4m3": lowbit.E4M3, "e8m0": lowbit.E8M0}[name]
    c = mlp_weights(make(blocks=3, F=704 if gated else 768, seed=21))
    W, n, B, H, d = quantise_weights(c, fmt, ("w_qkv", "w_o", "w_1", "w_2")), c["n"], c["B"], c["H"], c["d"]
    C = H * d
    kw = dict(weights4=name, activation_exponent=exponent, log_steps=2, forced_boundary=1)
    sizes = (c["blocks"], B, H, d, n["text"], n["ref"], n["tgt"], float("inf"), 10)
    ex = GatedDiTExecutor(*sizes, c["pos"], AXES, c["F"], **kw) if gated else DiTExecutor(*sizes, mlp_width=c["F"], **kw)
    first = {"text": 0, "ref": n["text"], "tgt": n["text"] + n["ref"]}

    def turned(x, r):
        """[B, H, n, d] by the positions of role r's rows in text, reference, target order."""
        if gated:
            return layers.rope_axes(x, c["pos"].double().cpu().numpy()[first[r]:first[r] + n[r]], AXES)
        return oracle_dit.apply_rope(x, np.arange(first[r], first[r] + n[r]))

    def places(t, b, r):
        """Where the block keeps the role's q, k and v."""
        if r == "ref":
            return ex.q_ref, ex.cache_k[b], ex.cache_v[b]
        return ex.qkv["text"][0] if r == "text" else ex.q_tgt[t % 2, b], ex.qkv[r][1], ex.qkv[r][2]

    rows, before, seen = [], {}, set()
    quant = dit.api.refadapt_quant4

    def recorded(segs, *args, **k):
        rows[:] = [s["x"].clone() for s in segs]
        return quant(segs, *args, **k)

    def check(phase, kind, t, b):
        if not kind.startswith("qkv"):
            return
        roles = ("ref",) if kind == "qkv_ref" else ("text", "tgt")
        if phase == "pre":
            before.update({r: [z.clone() for z in places(t, b, r)] for r in roles})
            return
        torch.cuda.synchronize()
        for r, x in zip(roles, rows):
            stream = STREAM_OF[r]
            plain, given = c["W"][b][stream], W[b][stream]["w_qkv"]
            w = lowbit.rounded(f64(plain["w_qkv"]), fmt, given.exponent)
            for s in range(B):
                mode = int(ex.modes[t % 2, b, s]) if r == "ref" else FULL
                seen.add((r, mode))
                p = lowbit.rounded(f64(x[s]), fmt, exponent)
                y = p @ w.T + plain["b_qkv"].double().cpu().numpy()
                e = C * 2.0 ** -23 * (np.abs(p) @ np.abs(w).T) + F32 * np.abs(y)
                y, e = (a.reshape(n[r], 3, H, d).transpose(1, 2, 0, 3) for a in (y, e))
                live = {REUSE: "", BOUNDARY: "q", COMPUTE: "qkv", FULL: "qkv"}[mode]
                for i, z in enumerate("qkv"):
                    got, was = places(t, b, r)[i][s], before[r][i][s]
                    if z not in live:
                        assert torch.equal(got, was), (t, b, r, z)
                        continue
                    ref, tol = y[i], BF * np.abs(y[i]) + e[i]
                    if z != "v":
                        norm = plain[z + "_norm"].double().cpu().numpy()
                        rms = np.sqrt((y[i] ** 2).mean(-1, keepdims=True) + 1e-6)
                        h = y[i] / rms * norm
                        top = np.abs(h).max(-1, keepdims=True)
                        ref = turned(h[None], r)[0]
                        tol = BF * np.abs(ref) + 2 * e[i].max(-1, keepdims=True) / rms * (np.abs(norm).max() + top) + 4 * F32 * top
                    within(got, ref, tol + 1e-30)

    monkeypatch.setattr(dit.api, "refadapt_quant4", recorded)
    ex.gemm_hook = check
    for t in range(2):
        ex.step(t, c["h_in"][t], lambda t, b: c["mods"][b], lambda b: W[b])
    ex.check()
    assert {m for r, m in seen if r == "ref"} == {REUSE, BOUNDARY, COMPUTE, FULL}
