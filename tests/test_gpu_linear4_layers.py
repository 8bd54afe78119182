"""The 4-bit products and the optimiser as a user has them: training.linear4 and
training.AdamW in torch's graph, DiTExecutor and GatedDiTExecutor with 4-bit weights,
captured steps, other streams, a wait that runs out, and the training example.

Each product of an executor's step is compared on the rows that it was given, as in
test_gpu_linear4 (exact 4-bit operands, K 2^-23 sum |a w| for the fp32 sums, half a bf16 step)."""
import math
import os
import sys

import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import lowbit
from test_gpu_gated_block import AXES, make
from test_gpu_linear4 import bf, within

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8


def api():
    from paper_2609_32415_gb300 import api as a
    return a


# ------------------------------------------------------------------ the autograd function
@pytest.mark.parametrize("fmt, exps", [(lowbit.E8M0, (0, 0)), (lowbit.E4M3, (1, -5))])
def test_linear4_is_the_two_calls(cuda_ok, fmt, exps):
    """Forward: Q(x) Q(w)^T; gradients: what refadapt_linear4_backward gives for the gradient that arrives."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(2)
    x, w = bf((2, 37, 192), g).requires_grad_(True), bf((128, 192), g, 0.07).requires_grad_(True)
    y = training.linear4(x, w, fmt, *exps)
    p, q = lowbit.rounded(f64(x.reshape(-1, 192)), fmt, exps[0]), lowbit.rounded(f64(w), fmt, exps[1])
    ref = p @ q.T
    within(y.reshape(-1, 128), ref, BF * np.abs(ref) + 192 * 2.0 ** -23 * (np.abs(p) @ np.abs(q).T) + 1e-30)
    given = []
    y.register_hook(lambda v: given.append(v.clone()))
    (y.transpose(1, 2) * bf((2, 128, 37), g)).float().sum().backward()  # arrives transposed
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    api().refadapt_linear4_backward(given[0].contiguous(), x, w, api().linear4_backward_workspace(2, 37, 192, 128), dx=dx,
                                    dw=dw)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)


def test_linear4_gradient_against_differences(cuda_ok):
    """The gradient is the formula's up to 4-bit rounding: each operand's error is independent of the other, at most
    a sixth of a value (a step of 2 at 4 to 6, half of it, over 5) and about 0.1 of the rows' norm, so the products'
    normwise error is below 0.1 sqrt(2) < 0.2; a difference of the loss along a random direction likewise."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(3)
    x, w, up = bf((1, 256, 256), g), bf((256, 256), g, 0.06), bf((1, 256, 256), g)
    xr, wr = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    (training.linear4(xr, wr) * up).float().sum().backward()
    for got, want in ((xr.grad, up.double() @ w.double()), (wr.grad, up[0].double().T @ x[0].double())):
        assert float((got.double() - want).norm() / want.norm()) < 0.2
    step = bf((1, 256, 256), g)
    loss = [float((training.linear4((x + s * step).to(torch.bfloat16), w).double() * up.double()).sum()) for s in (0.5, -0.5)]
    along = float((xr.grad.double() * step.double()).sum())
    # both are sums of 65536 products whose errors of 0.1 to 0.2 add up at random
    size = float(step.double().norm() * (up.double() @ w.double()).norm()) / math.sqrt(step.numel())
    assert abs(loss[0] - loss[1] - along) < 5 * 0.3 * size


def test_linear4_once_and_frozen(cuda_ok):
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(4)
    x, w = bf((1, 64, 128), g).requires_grad_(True), bf((64, 128), g, 0.1)
    (dx,) = torch.autograd.grad(training.linear4(x, w).float().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        dx.float().square().sum().backward()
    training.linear4(x, w).float().sum().backward()
    assert w.grad is None and x.grad is not None
    with torch.no_grad():
        assert not training.linear4(x, w).requires_grad
    empty = torch.empty((2, 0, 128), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    wr = w.clone().requires_grad_(True)
    training.linear4(empty, wr).float().sum().backward()
    assert bool((wr.grad == 0).all()) and empty.grad.shape == empty.shape


def test_backward_in_a_graph_beside_eager_ones(cuda_ok):
    """A captured forward and backward pass whose leaves no eager graph holds: the eager gradients."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(5)
    x, w, up = bf((2, 100, 256), g), bf((128, 256), g, 0.06), bf((2, 100, 128), g)

    def run(x, w):
        y = training.linear4(x, w)
        return (y, *torch.autograd.grad(y, (x, w), up))

    eager = [t.detach().clone() for t in run(x.clone().requires_grad_(True), w.clone().requires_grad_(True))]
    xs, ws = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = run(xs, ws)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, eager):
        assert torch.equal(a, b)


def test_on_another_stream(cuda_ok):
    a, g = api(), torch.Generator().manual_seed(6)
    x0, w0 = torch.randn((1, 300, 512), generator=g).pin_memory(), torch.randn((256, 512), generator=g) * 0.04

    def run(stream):
        with torch.cuda.stream(stream):
            x, w = x0.cuda(non_blocking=True).to(torch.bfloat16), w0.cuda().to(torch.bfloat16)
            codes, scales = a.quant4_buffers(1, 300, 512, lowbit.E8M0)
            out, dw = torch.empty((1, 300, 256), dtype=torch.bfloat16, device="cuda"), torch.empty_like(w)
            ws, norm, nws = a.linear4_backward_workspace(1, 300, 512, 256), torch.empty(2, device="cuda"), a.grad_norm_workspace()
            p, m = torch.zeros(w.numel(), device="cuda"), a.adamw_moments(torch.empty(w.numel(), device="cuda"), 8)
        w4 = a.weight4(w, lowbit.E8M0, stream=stream)
        torch.cuda._sleep(1000000)  # the current stream is busy with something else
        a.refadapt_quant4([{"x": x, "codes": codes, "scales": scales}], 512, lowbit.E8M0, stream=stream)
        a.refadapt_gemm4([{"a": codes, "a_scales": scales, "w": w4.codes, "w_scales": w4.scales, "out": out}], 256, 512, 0,
                         lowbit.E8M0, stream=stream)
        a.refadapt_linear4_backward(out, x, w, ws, dw=dw, stream=stream)
        a.refadapt_grad_norm([dw], 1.0, norm, nws, stream=stream)
        a.refadapt_adamw([{"p": p, "g": dw.view(-1), **m}], 1e-3, 1, grad_scale=norm[1:], stream=stream)
        stream.synchronize()
        return out.clone(), dw.clone(), norm.clone(), p.clone()

    for s, t in zip(run(torch.cuda.current_stream()), run(torch.cuda.Stream())):
        assert torch.equal(s, t)


# ------------------------------------------------------------------ the executors
def quantise_weights(c, fmt, names):
    return [{st: {k: api().weight4(v, fmt) if k in names else v for k, v in w.items()} for st, w in blk.items()}
            for blk in c["W"]]


def mlp_weights(c):
    """make()'s weights as DiTExecutor's: an MLP in place of the gated feed-forward."""
    g = torch.Generator().manual_seed(77)
    C, F = c["H"] * c["d"], c["F"]
    for w in c["W"]:
        for st in w.values():
            st.update(w_1=bf((F, C), g, C ** -0.5), b_1=torch.zeros(F, device="cuda"))
    return c


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", ["e4m3", "e8m0"])
def test_executor_products(cuda_ok, monkeypatch, gated, name):
    """Two steps (all rows, then what the gate decides): every product of the executor, on the rows it was given."""
    from paper_2609_32415_gb300 import DiTExecutor, GatedDiTExecutor, dit
    a, fmt = api(), {"e4m3": lowbit.E4M3, "e8m0": lowbit.E8M0}[name]
    c = mlp_weights(make(blocks=2, F=704 if gated else 768, seed=11))
    W = quantise_weights(c, fmt, ("w_qkv", "w_o", "w_1", "w_2"))
    n = c["n"]
    kw = dict(weights4=name, log_steps=2)
    ex = GatedDiTExecutor(c["blocks"], c["B"], c["H"], c["d"], n["text"], n["ref"], n["tgt"], 0.05, 5, c["pos"], AXES, c["F"],
                          **kw) if gated else \
        DiTExecutor(c["blocks"], c["B"], c["H"], c["d"], n["text"], n["ref"], n["tgt"], 0.05, 5, mlp_width=c["F"], **kw)
    seen = []
    rows, product = a.refadapt_quant4, a.refadapt_gemm4

    def quant(segs, C, f, mode=None, stream=None):
        rows(segs, C, f, mode=mode, stream=stream)
        seen.append([s["x"].clone() for s in segs])

    def gemm(segs, N, K, epi, f, mode=None, **k):
        before = [{z: s[z].clone() for z in ("out", "resid") if z in s} for s in segs]
        product(segs, N, K, epi, f, mode=mode, **k)
        torch.cuda.synchronize()
        live = [m != 0 for m in mode.tolist()] if mode is not None else None
        for s, x, was in zip(segs, seen.pop(), before):
            if epi == 3:
                continue  # its epilogue is checked in test_gpu_linear4
            w = lowbit.values(*weight_of(s["w"], s["w_scales"], f), f, s["w_exponent"])
            for b in range(x.shape[0]):
                if s.get("gated") and not live[b]:
                    assert torch.equal(s["out"][b], was["out"][b])
                    continue
                p = lowbit.rounded(f64(x[b]), f, s["a_exponent"])
                y = p @ w.T + s["bias"].double().cpu().numpy()
                tol = K * 2.0 ** -23 * (np.abs(p) @ np.abs(w).T) + 2.0 ** -16 * np.abs(y)
                if epi == 1:
                    y = y / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))
                    tol = 1.2 * tol
                elif epi == 2:
                    gate = s["gate"][b].double().cpu().numpy()
                    y, tol = f64(was["resid"][b]) + gate * y, np.abs(gate) * tol
                within(s["out"][b], y, tol + BF * np.abs(y) + 1e-30)

    monkeypatch.setattr(dit.api, "refadapt_quant4", quant)
    monkeypatch.setattr(dit.api, "refadapt_gemm4", gemm)
    for t in range(2):
        ex.step(t, c["h_in"][t], lambda t, b: c["mods"][b], lambda b: W[b])
    ex.check()
    assert not seen and set(np.unique(ex.modes.cpu().numpy())) - {3}
    with pytest.raises(ValueError, match="Weight4"):
        ex.step(0, c["h_in"][0], lambda t, b: c["mods"][b], lambda b: c["W"][b])


def weight_of(codes, scales, f):
    c = codes.cpu().numpy()
    full = np.zeros((c.shape[0], 2 * c.shape[1]), np.int64)
    full[:, 0::2], full[:, 1::2] = c & 15, c >> 4
    return full, lowbit.untile(scales.cpu().numpy(), c.shape[0], -(-full.shape[1] // lowbit.BLOCK[f]))


def test_executor_replays_as_a_graph(cuda_ok):
    from paper_2609_32415_gb300 import GatedDiTExecutor
    c = make(blocks=2, seed=9)
    W, n = quantise_weights(c, lowbit.E4M3, ("w_qkv", "w_o", "w_2")), c["n"]
    eager, ex = (GatedDiTExecutor(c["blocks"], c["B"], c["H"], c["d"], n["text"], n["ref"], n["tgt"], 0.05, 5, c["pos"], AXES,
                                  c["F"], weights4="e4m3") for _ in range(2))
    args = (lambda t, b: c["mods"][b], lambda b: W[b])
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


def test_unknown_format_is_refused(cuda_ok):
    from paper_2609_32415_gb300 import DiTExecutor
    with pytest.raises(ValueError, match="weights4"):
        DiTExecutor(1, 1, 4, 64, 8, 8, 8, 0.1, 5, weights4="int4")


# ------------------------------------------------------------------ a wait that runs out
@pytest.mark.parametrize("epilogue", [0, 3])
@pytest.mark.parametrize("tile_mode", [1, 2])
def test_a_wait_that_runs_out(cuda_ok, tile_mode, epilogue):
    """One output tile with a K so long that the epilogue gives up while loads and MMAs go on (see
    test_gpu_gemm_timeout): they land, the error word is set, and the next call gives what the first gave."""
    from paper_2609_32415_gb300._lib import RA_ETIMEOUT, RefAdaptError
    a, n, K = api(), 256, 65536
    N = 256 if epilogue == 0 else 768
    codes, w = (torch.randint(0, 256, s, dtype=torch.uint8, device="cuda") for s in ((1, n, K // 2), (N, K // 2)))
    scales = [torch.full((a.refadapt_quant4_scales_size(r, K, 1),), 120, dtype=torch.uint8, device="cuda") for r in (n, N)]
    seg = {"a": codes, "a_scales": scales[0], "w": w, "w_scales": scales[1]}
    kw = {}
    if epilogue == 0:
        seg["out"] = torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda")
        outs = [seg["out"]]
    else:
        seg.update({z: torch.empty((1, 4, n, 64), dtype=torch.bfloat16, device="cuda") for z in "qkv"},
                   q_norm=torch.ones(64, device="cuda"), k_norm=torch.ones(64, device="cuda"))
        outs = [seg[z] for z in "qkv"]
        kw = dict(rope=a.rope_table(n, 64), H=4, d=64)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        a.refadapt_gemm4([seg], N, K, epilogue, 1, err_word=err, tile_mode=tile_mode, **kw)

    call()
    a.refadapt_check_error(err)
    want = [o.clone() for o in outs]
    a.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(3):
            call()
            with pytest.raises(RefAdaptError) as e:
                a.refadapt_check_error(err)
            assert e.value.status == RA_ETIMEOUT
    finally:
        a.refadapt_set_wait_budget_ns(500_000_000)
    call()
    a.refadapt_check_error(err)
    for o, v in zip(outs, want):
        assert torch.equal(o, v)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tile_mode", [1, 2])
def test_a_wait_that_runs_out_before_other_tiles(cuda_ok, tile_mode, d):
    """The same with several tiles to a CTA, whose epilogue warps take turns and, for heads of 128, meet: those
    that did not give up wait for no one."""
    from paper_2609_32415_gb300._lib import RA_ETIMEOUT, RefAdaptError
    a, n, K, N = api(), 128 * 70, 65536, 768
    g = torch.Generator(device="cuda").manual_seed(d)
    codes, w = (torch.randint(0, 256, s, dtype=torch.uint8, device="cuda", generator=g) for s in ((1, n, K // 2), (N, K // 2)))
    scales = [torch.full((a.refadapt_quant4_scales_size(r, K, 1),), 120, dtype=torch.uint8, device="cuda") for r in (n, N)]
    outs = [torch.empty((1, N // 3 // d, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    seg = {"a": codes, "a_scales": scales[0], "w": w, "w_scales": scales[1], "q": outs[0], "k": outs[1], "v": outs[2],
           "q_norm": torch.ones(d, device="cuda"), "k_norm": torch.ones(d, device="cuda")}
    err, rope = torch.zeros(1, dtype=torch.int32, device="cuda"), a.rope_table(n, d)

    def call():
        a.refadapt_gemm4([seg], N, K, 3, 1, err_word=err, tile_mode=tile_mode, rope=rope, H=N // 3 // d, d=d)

    call()
    a.refadapt_check_error(err)
    want = [o.clone() for o in outs]
    a.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(3):
            call()
            with pytest.raises(RefAdaptError) as e:
                a.refadapt_check_error(err)
            assert e.value.status == RA_ETIMEOUT
    finally:
        a.refadapt_set_wait_budget_ns(500_000_000)
    call()
    a.refadapt_check_error(err)
    for o, v in zip(outs, want):
        assert torch.equal(o, v)


# ------------------------------------------------------------------ the optimiser
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_class(cuda_ok, bits):
    """Three steps of the class are three pairs of calls; bf16 parameters are the rounding of their fp32 copies; a
    parameter without a gradient stays; a saved state goes on in another one."""
    from paper_2609_32415_gb300 import training
    a, g = api(), torch.Generator().manual_seed(14)
    make_params = lambda: [torch.nn.Parameter(p.clone()) for p in start]  # noqa: E731
    start = [bf((37, 65), g), torch.randn(100, generator=g).cuda(), bf((64,), g), torch.randn(3, generator=g).cuda()]
    grads = [[torch.randn(p.shape, generator=g).to(p.dtype).cuda() for p in start] for _ in range(4)]
    params = make_params()
    opt = training.AdamW(params, 1e-2, bits=bits, max_norm=5.0, seed=3)
    mine = [{"p": p.detach().float().clone(), **a.adamw_moments(p, bits)} for p in start[:3]]
    norm, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    for k in range(3):
        opt.zero_grad()
        for p, v in zip(params[:3], grads[k]):
            p.grad = v.clone()
        opt.step()
        a.refadapt_grad_norm(grads[k][:3], 5.0, norm, ws)
        a.refadapt_adamw([{**m, "g": v} for m, v in zip(mine, grads[k])], 1e-2, k + 1, grad_scale=norm[1:], seed=3)
        assert torch.equal(opt.norm, norm) and float(norm[1]) < 1.0
        for p, m in zip(params, mine):
            assert torch.equal(p.detach(), m["p"].to(p.dtype))
    assert torch.equal(params[3].detach(), start[3])
    other_params = [torch.nn.Parameter(p.detach().clone()) for p in params]
    other = training.AdamW(other_params, 1e-2, bits=bits, max_norm=5.0, seed=3)
    other.load_state_dict(opt.state_dict())
    for o, ps in ((opt, params), (other, other_params)):
        for p, v in zip(ps[:3], grads[3]):
            p.grad = v.t().contiguous().t() if v.dim() == 2 else v  # a gradient that is not contiguous
        o.step()
    for p, q in zip(params, other_params):
        assert torch.equal(p.detach(), q.detach())


def test_adamw_class_refuses(cuda_ok):
    from paper_2609_32415_gb300 import training
    p = torch.nn.Parameter(torch.zeros(4, 6, device="cuda"))
    for bad, text in (([], "no parameters"), ([p, p], "twice"), ([p.t()], "contiguous"), ([p.half()], "fp32 or bf16"),
                      ([torch.zeros(3)], "CUDA")):
        with pytest.raises(ValueError, match=text):
            training.AdamW(bad, 1e-3)
    with pytest.raises(ValueError, match="32 or 8"):
        training.AdamW([p], 1e-3, bits=16)
    with pytest.raises(ValueError, match="bits"):
        training.AdamW([p], 1e-3, bits=8).load_state_dict(training.AdamW([p], 1e-3).state_dict())


def test_a_captured_training_step(cuda_ok):
    """Forward, backward and the optimiser's step in one graph, replayed: the eager steps' parameters."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(15)
    x, up, w = bf((2, 100, 256), g), bf((2, 100, 128), g), bf((128, 256), g, 0.06)

    def step(p, opt):
        p.grad = torch.autograd.grad(training.linear4(x, p), p, up)[0]
        opt.step()

    eager = torch.nn.Parameter(w.clone())
    opt = training.AdamW([eager], 1e-2, bits=8, max_norm=1.0, capturable=True)
    for _ in range(3):
        step(eager, opt)
    p = torch.nn.Parameter(w.clone())
    opt2 = training.AdamW([p], 1e-2, bits=8, max_norm=1.0, capturable=True)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(p, opt2)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(opt2.count) == 3 and torch.equal(p.detach(), eager.detach())


@pytest.mark.parametrize("bits", [8, 32])
def test_training_example_runs(cuda_ok, bits):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_gated_block
    losses = train_gated_block.train(steps=4, height=9, width=11, linear4=True, bits=bits)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
