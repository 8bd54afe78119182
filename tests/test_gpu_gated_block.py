"""The gated block's layers as they are used together: GatedDiTExecutor against
an fp64 loop over the same inputs (all four modes), its capture as a CUDA graph,
the autograd functions against torch's own gradients in fp64, the training
example, and calls on another stream than torch's current one.

Tolerances of the stack: those of the DiT stack's closed loop (each block adds
the attention path's error of about 1e-3 and single-step bf16 differences of its
layers): 3e-2 of (|r| + rms) per element, 1e-2 normwise."""
import math
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from _helpers import ROLES, f64, o_close
from oracle import COMPUTE, FULL, REUSE, dit, layers

pytestmark = pytest.mark.gpu
STREAM_OF = {"text": "text", "ref": "image", "tgt": "image"}
KINDS = {"none": 0, "layer": 1, "rms": 2}
AXES = (16, 24, 24)


def make(B=2, H=4, d=64, n=(21, 130, 77), blocks=3, F=704, seed=0, weights=True):
    g = torch.Generator().manual_seed(seed)
    C = H * d

    def bf(*s, scale=1.0):
        return (torch.randn(s, generator=g) * scale).to(torch.bfloat16).cuda()

    def f32(*s, scale=1.0, mean=0.0):
        return (torch.randn(s, generator=g) * scale + mean).cuda()

    W, mods = [], []
    for _ in range(blocks):
        w, m = {}, {}
        for st in ("text", "image"):
            w[st] = {"w_qkv": bf(3 * C, C, scale=C ** -0.5), "b_qkv": f32(3 * C, scale=0.02),
                     "q_norm": f32(d, scale=0.1, mean=1.0), "k_norm": f32(d, scale=0.1, mean=1.0),
                     "w_o": bf(C, C, scale=C ** -0.5), "b_o": f32(C, scale=0.02), "w_gate": bf(F, C, scale=C ** -0.5),
                     "w_up": bf(F, C, scale=C ** -0.5), "w_2": bf(C, F, scale=F ** -0.5), "b_2": f32(C, scale=0.02)}
            if weights:
                w[st].update({k: f32(C, scale=0.1, mean=1.0) for k in ("pre_a", "post_a", "pre_m", "post_m")})
            m[st] = {k: f32(B, C, scale=0.1) for k in ("shift_a", "scale_a", "shift_m", "scale_m")}
            m[st].update({k: f32(B, C, scale=0.05, mean=0.3) for k in ("gate_a", "gate_m")})
        W.append(w)
        mods.append(m)
    N = dict(zip(ROLES, n))
    h_in = [{r: bf(B, N[r], C) for r in ROLES} for _ in range(2)]
    for r in ("text", "ref"):
        h_in[1][r] = h_in[0][r]
    pos = torch.randint(-20, 20, (sum(n), 3), generator=g).float().cuda()
    return dict(B=B, H=H, d=d, n=N, blocks=blocks, F=F, W=W, mods=mods, h_in=h_in, pos=pos)


def oracle_loop(c, modes, pre, post, act, eps=1e-6):
    """The stack's rows per step for given modes [t][b][s]."""
    B, H, d, C = c["B"], c["H"], c["d"], c["H"] * c["d"]
    rb, pos = dit.round_bf16, c["pos"].double().cpu().numpy()
    at = {"text": 0, "ref": c["n"]["text"], "tgt": c["n"]["text"] + c["n"]["ref"]}
    cache = [[None] * B for _ in range(c["blocks"])]
    hbar = [[None] * B for _ in range(c["blocks"] + 1)]
    outs = []

    def vec(x):
        return None if x is None else x.double().cpu().numpy()

    def norm_in(h, m, w, k, s):
        x = layers.normalise(KINDS[pre], h, eps)[0]
        if w.get("pre_" + k) is not None:
            x = x * vec(w["pre_" + k])
        return rb(x * (1 + vec(m["scale_" + k])[s]) + vec(m["shift_" + k])[s])

    def after(h, y, m, w, k, s):
        z = layers.normalise(KINDS[post], y, eps)[0]
        if w.get("post_" + k) is not None:
            z = z * vec(w["post_" + k])
        return h + vec(m["gate_" + k])[s] * z  # not rounded yet

    def qkv(x, w, r):
        y = dit.linear(x, f64(w["w_qkv"]), vec(w["b_qkv"]))
        q, k, v = (y[:, i * C:(i + 1) * C].reshape(-1, H, d).transpose(1, 0, 2) for i in range(3))
        p = pos[at[r]:at[r] + c["n"][r]]
        q = layers.rope_axes(dit.rms_norm(q, vec(w["q_norm"]), eps)[None], p, AXES)[0]
        k = layers.rope_axes(dit.rms_norm(k, vec(w["k_norm"]), eps)[None], p, AXES)[0]
        return rb(q), rb(k), rb(v)

    def finish(h, o, m, w, s):
        y = rb(dit.linear(rb(o).transpose(1, 0, 2).reshape(-1, C), f64(w["w_o"]), vec(w["b_o"])))
        h1 = after(h, y, m, w, "a", s)
        x = norm_in(h1, m, w, "m", s)
        u = rb(layers.glu(x, f64(w["w_gate"]), f64(w["w_up"]), act)[0])
        y = rb(dit.linear(u, f64(w["w_2"]), vec(w["b_2"])))
        return after(rb(h1), y, m, w, "m", s)

    for t, h_in in enumerate(c["h_in"]):
        cur = {r: [f64(h_in[r])[s] for s in range(B)] for r in ("text", "tgt")}  # not rounded between blocks' norms
        for s in range(B):
            hbar[0][s] = f64(h_in["ref"])[s]
        for b in range(c["blocks"]):
            W, M = c["W"][b], c["mods"][b]
            for s in range(B):
                mode = modes[t][b][s]
                p = {}
                for r in ("text", "tgt"):
                    w, m = W[STREAM_OF[r]], M[STREAM_OF[r]]
                    p[r] = qkv(norm_in(cur[r][s], m, w, "a", s), w, r)
                w, m = W["image"], M["image"]
                q_ref = None
                if mode != REUSE:
                    q_ref, k_ref, v_ref = qkv(norm_in(hbar[b][s], m, w, "a", s), w, "ref")
                    if mode in (COMPUTE, FULL):
                        cache[b][s] = (k_ref, v_ref)
                kc, vc = cache[b][s]
                res = oracle.block_attention({"text": p["text"][0], "ref": q_ref, "tgt": p["tgt"][0]},
                                             {"text": p["text"][1], "ref": kc, "tgt": p["tgt"][1]},
                                             {"text": p["text"][2], "ref": vc, "tgt": p["tgt"][2]}, mode,
                                             1 / math.sqrt(d))
                for r in ("text", "tgt"):
                    cur[r][s] = finish(rb(cur[r][s]), res["O"][r], M[STREAM_OF[r]], W[STREAM_OF[r]], s)
                if mode != REUSE:
                    hbar[b + 1][s] = rb(finish(hbar[b][s], res["O"]["ref"], m, w, s))
        outs.append({"text": np.stack([rb(x) for x in cur["text"]]), "tgt": np.stack([rb(x) for x in cur["tgt"]]),
                     "hbar": [np.stack(x) for x in hbar]})
    return outs


def executor(c, pre, post, act, forced=1):
    from paper_2609_32415_gb300 import GatedDiTExecutor
    return GatedDiTExecutor(c["blocks"], c["B"], c["H"], c["d"], *(c["n"][r] for r in ROLES), float("inf"), 10,
                            c["pos"], AXES, c["F"], pre=pre, post=post, act=act, forced_boundary=forced, log_steps=2)


@pytest.mark.parametrize("pre,post,act,weights", [("rms", "rms", "silu", True), ("layer", "rms", "gelu", False),
                                                  ("rms", "none", "silu", False)])
def test_gated_stack_closed_loop(cuda_ok, pre, post, act, weights):
    c = make(seed=len(pre) + len(post), weights=weights)
    ex = executor(c, pre, post, act)
    outs = []
    for t in range(2):
        ex.step(t, c["h_in"][t], lambda t, b: c["mods"][b], lambda b: c["W"][b])
        torch.cuda.synchronize()
        outs.append({"text": f64(ex.h["text"]), "tgt": f64(ex.h["tgt"]), "hbar": [f64(x) for x in ex.hbar]})
    ex.check()
    modes = ex.modes.cpu().numpy()
    assert (modes[0] == FULL).all() and [list(m) for m in modes[1]] == [[0, 0], [1, 1], [2, 2]]
    ref = oracle_loop(c, modes, pre, post, {"silu": 0, "gelu": 1}[act])
    for t in range(2):
        for k, got, want in [(r, outs[t][r], ref[t][r]) for r in ("text", "tgt")] + \
                [("hbar%d" % b, outs[t]["hbar"][b], ref[t]["hbar"][b]) for b in range(c["blocks"] + 1)]:
            ok, worst, normwise = o_close(got, want, 3e-2)
            assert ok and normwise <= 1e-2, (t, k, worst, normwise)


def test_gated_stack_steps_replay_as_a_graph(cuda_ok):
    c = make(seed=9)
    eager, ex = executor(c, "rms", "rms", "silu"), executor(c, "rms", "rms", "silu")
    args = (lambda t, b: c["mods"][b], lambda b: c["W"][b])
    for t in range(2):
        eager.step(t, c["h_in"][t], *args)
    ex.step(0, c["h_in"][0], *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ex.step(1, c["h_in"][1], *args)
    graph.replay()
    torch.cuda.synchronize()
    ex.check()
    for r in ("text", "tgt"):
        assert torch.equal(ex.h[r], eager.h[r]), r


def test_unknown_options_are_refused(cuda_ok):
    c = make(blocks=1)
    for kw in ({"pre": "group"}, {"post": "x"}, {"act": "relu"}):
        with pytest.raises(ValueError, match="unknown"):
            executor(c, **dict({"pre": "rms", "post": "rms", "act": "silu"}, **kw))
    c["pos"] = c["pos"][:-1]
    with pytest.raises(ValueError, match="coordinates"):
        executor(c, "rms", "rms", "silu")


def relative(a, b):
    return float((a.double() - b).norm() / (b.norm() + 1e-300))


def test_autograd_functions_match_torch(cuda_ok):
    """The layers' gradients through torch's graph against fp64 autograd of the
    same expression: bf16 tensors between layers and bf16 gradients leave a few
    2^-9 normwise, 1e-2 has room; fp32 vectors' gradients inherit those inputs."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(4)
    B, n, C, F, H = 2, 45, 256, 448, 4

    def leaf(*s, scale=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(s, generator=g) * scale + mean).to(dtype).cuda().requires_grad_(True)

    h, y = leaf(B, n, C), leaf(B, n, C)
    wg, wu, wd = leaf(F, C, scale=C ** -0.5), leaf(F, C, scale=C ** -0.5), leaf(C, F, scale=F ** -0.5)
    f32 = dict(dtype=torch.float32)
    vec = {"gate": leaf(B, C, scale=0.1, mean=0.5, **f32), "scale": leaf(B, C, scale=0.1, **f32),
           "shift": leaf(B, C, scale=0.1, **f32), "post_w": leaf(C, scale=0.1, mean=1.0, **f32),
           "pre_w": leaf(C, scale=0.1, mean=1.0, **f32)}
    pos = torch.randn((n, 2), generator=g).cuda() * 10
    up_h, up_q = (torch.randn(s, generator=g).cuda() for s in ((B, n, C), (B, H, n, C // H)))

    def loss_here():
        h1, x = training.residual_norm(h, y, 2, 1, **vec)
        z = training.gated_feed_forward(x, wg, wu, wd, 0)
        q = training.rope_axes(z.unflatten(2, (H, -1)).transpose(1, 2), pos, (32, 32))
        return (h1.float() * up_h).sum() + (q.float() * up_q).sum()

    leaves = [h, y, wg, wu, wd, *vec.values()]
    got = torch.autograd.grad(loss_here(), leaves)
    wide = [t.detach().double().requires_grad_(True) for t in leaves]
    h2, y2, wg2, wu2, wd2, gate, scale, shift, post_w, pre_w = wide
    h1 = h2 + gate[:, None] * (y2 / ((y2 ** 2).mean(-1, keepdim=True) + 1e-6).sqrt() * post_w)
    m = h1 - h1.mean(-1, keepdim=True)
    x = m / ((m ** 2).mean(-1, keepdim=True) + 1e-6).sqrt() * pre_w * (1 + scale[:, None]) + shift[:, None]
    z = torch.nn.functional.silu(x @ wg2.T) * (x @ wu2.T) @ wd2.T
    q = z.unflatten(2, (H, -1)).transpose(1, 2)
    ang = torch.cat([pos[:, a:a + 1].double() * 10000.0 ** (-torch.arange(0, 32, 2, device="cuda").double() / 32)
                     for a in range(2)], -1)
    e, o, cs, sn = q[..., 0::2], q[..., 1::2], torch.cos(ang), torch.sin(ang)
    q = torch.stack((e * cs - o * sn, e * sn + o * cs), -1).flatten(-2)
    want = torch.autograd.grad((h1 * up_h).sum() + (q * up_q).sum(), wide)
    for name, a, b in zip(["h", "y", "wg", "wu", "wd", *vec], got, want):
        assert relative(a, b) < 1e-2, (name, relative(a, b))


def test_frozen_inputs_get_no_gradient(cuda_ok):
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(5)
    x, w, wd = ((torch.randn(s, generator=g) * 0.1).to(torch.bfloat16).cuda() for s in ((1, 20, 256), (128, 256), (256, 128)))
    wd.requires_grad_(True)
    training.gated_feed_forward(x, w, w, wd, 1).float().sum().backward()
    assert wd.grad is not None and x.grad is None and w.grad is None


def test_training_example_learns(cuda_ok):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_gated_block
    losses = train_gated_block.train(steps=40, height=9, width=11)
    assert all(math.isfinite(v) for v in losses)
    assert np.mean(losses[-5:]) < 0.7 * np.mean(losses[:5]), losses


def test_calls_on_another_stream(cuda_ok):
    """Every call runs on the stream that it is given: results on a side stream
    equal those on the current one, with inputs made on the side stream."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(6)
    x0, w0 = (torch.randn((1, 300, 512), generator=g)).pin_memory(), (torch.randn((2, 768, 512), generator=g) * 0.04)

    def run(stream):
        with torch.cuda.stream(stream):
            x = x0.cuda(non_blocking=True).to(torch.bfloat16)
            w = w0.to(torch.bfloat16).cuda()
            out, h, pos = torch.empty((1, 300, 768), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x), \
                torch.arange(300, device="cuda").float()[:, None].contiguous()
            q = x.view(1, 300, 8, 64).permute(0, 2, 1, 3)
            qo = torch.empty_like(q)
        torch.cuda._sleep(1000000)  # the current stream is busy with something else
        api.refadapt_residual_norm([{"h": x, "y": x, "h_out": h}], 512, 2, 0, stream=stream)
        api.refadapt_glu([{"x": h, "w_gate": w[0], "w_up": w[1], "out": out}], 768, 512, 0, stream=stream)
        api.refadapt_rope_axes([(q, qo)], pos, (64,), stream=stream)
        stream.synchronize()
        return h.clone(), out.clone(), qo.clone()

    for a, b in zip(run(torch.cuda.current_stream()), run(torch.cuda.Stream())):
        assert torch.equal(a, b)
