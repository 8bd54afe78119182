"""GPU parity of the gated block's layers (refadapt_rope_axes and its table,
refadapt_residual_norm and its backward pass) against the fp64 oracle
(oracle/layers.py) on the same inputs, and their refusals.

Tolerances. A bf16 output is one rounding of an fp32 value: half a unit in the
last place is at most 2^-8 |ref|, and the fp32 value is off by a few 2^-24 of the
magnitudes it is made of (`mag`), bounded by 2^-16 mag with room for a row's
statistics: |got - ref| <= 2^-8 |ref| (1 + 2^-6) + 2^-16 mag. An fp32 column sum
of n terms t adds at most 300 of them in one chain (rows of a CTA, then 32
slices): |got - ref| <= 320 * 2^-24 * sum |t|, of which the terms' own errors
(below 2^-20 |t|) are a small part."""
import math

import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import layers

pytestmark = pytest.mark.gpu


def bf(shape, g, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=g) * scale + mean).to(torch.bfloat16).cuda()


def f32(shape, g, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=g) * scale + mean).cuda()


def d64(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, ref, mag):
    err = np.abs(np.asarray(got, np.float64) - ref)
    tol = 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -6) + 2.0 ** -16 * mag
    return bool((err <= tol).all()), float((err / (tol + 1e-300)).max())


# ------------------------------------------------------------------ rotary positions
def heads(B, H, n, d, g, layout):
    if layout == "token":
        return bf((B, n, H, d), g).permute(0, 2, 1, 3)
    if layout == "wide":  # rows of a wider buffer, head-major
        return bf((B, H, n, d + 24), g)[..., 16:16 + d]
    return bf((B, H, n, d), g)


@pytest.mark.parametrize("B,H,Hk,n,d,axes,layout", [
    (1, 8, 8, 1, 64, (8, 28, 28), "token"),
    (2, 5, 1, 333, 64, (32, 32), "head"),
    (1, 24, 24, 1009, 128, (16, 56, 56), "head"),
    (2, 16, 4, 77, 128, (44, 44, 40), "token"),
    (3, 3, 2, 130, 96, (32, 16), "wide"),      # columns past the axes are copied
    (1, 2, 2, 40, 256, (2, 2, 2, 250), "token"),
    (1, 1, 1, 5, 8, (6,), "head"),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_axes(cuda_ok, B, H, Hk, n, d, axes, layout, inverse):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(n * d + H)
    q, k = heads(B, H, n, d, g, layout), heads(B, Hk, n, d, g, layout)
    per_sample = B > 1 and n % 2 == 1
    pos = (torch.randint(-300, 300, (B, n, len(axes)) if per_sample else (n, len(axes)), generator=g).float()
           + 0.25).cuda()
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    api.refadapt_rope_axes([(q, qo), (k, ko)], pos, axes, inverse=inverse)
    torch.cuda.synchronize()
    for x, y in ((q, qo), (k, ko)):
        ref = layers.rope_axes(f64(x), d64(pos), axes, inverse=inverse)
        ok, worst = close(f64(y), ref, np.abs(f64(x)).max())
        assert ok, worst
        m = sum(axes)
        assert torch.equal(y[..., m:], x[..., m:])
    # in place, one tensor
    z = q.clone()
    api.refadapt_rope_axes([(z, z)], pos, axes, inverse=inverse)
    assert torch.equal(z, qo)


def test_rope_axes_far_positions_and_infinities(cuda_ok):
    """Angles of many turns stay good to fp32, copied columns keep infinities
    and NaN, turned pairs with one spread it inside the pair only."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(5)
    x = bf((1, 2, 64, 64), g)
    pos = torch.linspace(-2.0 ** 22, 2.0 ** 22, 64).reshape(64, 1).round().cuda()
    x[0, 0, 3, 40] = float("inf")
    x[0, 1, 5, 63] = float("nan")
    x[0, 0, 7, 0] = float("inf")
    y = torch.empty_like(x)
    api.refadapt_rope_axes([(x, y)], pos, (32,))
    got, xx = f64(y), f64(x)
    assert got[0, 0, 3, 40] == np.inf and np.isnan(got[0, 1, 5, 63])
    assert not np.isfinite(got[0, 0, 7, :2]).any()
    xx[0, 0, 3, 40] = xx[0, 1, 5, 63] = xx[0, 0, 7, 0] = 0.0
    ref = layers.rope_axes(xx, d64(pos), (32,))
    for at in ((0, 0, 3, 40), (0, 1, 5, 63), (0, 0, 7, 0), (0, 0, 7, 1)):
        got[at] = ref[at]
    ok, worst = close(got, ref, np.abs(xx).max())
    assert ok, worst


def test_rope_axes_table_feeds_the_qkv_epilogue(cuda_ok):
    """The table against the angles, and a QKV projection with it against a
    projection with the one-axis table of the same angles."""
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RA_EPI_QKV
    t, hh, ww = 3, 5, 7
    pos = torch.stack(torch.meshgrid(torch.arange(t), torch.arange(hh) - 2, torch.arange(ww) - 3, indexing="ij"),
                      -1).reshape(-1, 3).float().cuda()
    axes = (16, 24, 24)
    table = api.rope_axes_table(pos, 64, axes)
    ang = layers.rope_axes_angles(d64(pos), axes)
    assert np.abs(d64(table[..., 0]) - np.cos(ang)).max() < 1e-6
    assert np.abs(d64(table[..., 1]) - np.sin(ang)).max() < 1e-6
    part = api.rope_axes_table(pos, 64, (16, 24, 8))
    assert torch.equal(part[:, 24:, 0], torch.ones_like(part[:, 24:, 0])) and not part[:, 24:, 1].any()
    g = torch.Generator().manual_seed(2)
    H, d, n = 4, 64, t * hh * ww
    C = H * d
    x, w = bf((1, n, C), g), bf((3 * C, C), g, C ** -0.5)
    ones = torch.ones(d, device="cuda")

    def project(rope):
        out = [torch.empty((1, H, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        api.refadapt_gemm([{"a": x, "w": w, "q": out[0], "k": out[1], "v": out[2], "q_norm": ones, "k_norm": ones}],
                          3 * C, C, RA_EPI_QKV, rope=rope, H=H, d=d)
        return out

    q, k, v = project(table)
    flat = torch.zeros_like(table)
    flat[..., 0] = 1.0
    q0, k0, v0 = project(flat)
    # q0 is rounded to bf16 before it is turned here, so both roundings count
    for a, b in ((q, q0), (k, k0)):
        ref = layers.rope_axes(f64(b), d64(pos), axes)
        err = np.abs(f64(a) - ref)
        assert (err <= 2.0 ** -7 * (np.abs(f64(b)).max() + np.abs(ref))).all()
    assert torch.equal(v, v0)


def test_rope_axes_refusals(cuda_ok):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RefAdaptError
    x = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((4, 2), device="cuda")
    for axes, msg in (((3, 4), "even"), ((64, 64), "columns"), ((0, 4), "even")):
        with pytest.raises(RefAdaptError, match=msg):
            api.refadapt_rope_axes([(x, x)], pos, axes)
    with pytest.raises(RefAdaptError, match="base"):
        api.refadapt_rope_axes([(x, x)], pos, (4, 4), base=1.0)
    with pytest.raises(ValueError, match="pos"):
        api.refadapt_rope_axes([(x, x)], pos[:3], (4, 4))
    with pytest.raises(ValueError, match="one shape"):
        api.refadapt_rope_axes([(x, x[:, :1])], pos, (4, 4))
    odd = torch.zeros((1, 2, 4, 72), dtype=torch.bfloat16, device="cuda")[..., 1:65]
    with pytest.raises(RefAdaptError, match="aligned"):
        api.refadapt_rope_axes([(odd, odd)], pos, (4, 4))
    empty = torch.zeros((1, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    api.refadapt_rope_axes([(empty, empty)], pos[:0], (4, 4))
    with pytest.raises(ValueError, match="table"):
        api.refadapt_rope_axes_table(torch.zeros((3, 32, 2), device="cuda"), pos, (4, 4))


# ------------------------------------------------------------------ norms around a branch
def norm_case(B, n, C, g, weights, wide=False, mod=True):
    def rows(scale, mean):
        if not wide:
            return bf((B, n, C), g, scale, mean)
        return bf((B, n + 3, C + 40), g, scale, mean)[:, 2:2 + n, 24:24 + C]
    s = {"h": rows(2.0, 0.3), "y": rows(1.5, -0.7)}
    if mod:
        s.update(gate=f32((B, C), g, 0.3, 0.5), scale=f32((B, C), g, 0.1), shift=f32((B, C), g, 0.1))
    if weights:
        s.update(post_w=f32((C,), g, 0.1, 1.0), pre_w=f32((C,), g, 0.1, 1.0))
    return s


def vectors(s, *names):
    return {k: d64(s.get(k)) for k in names}


def check_forward(s, post, pre, eps, alpha, skip=()):
    y = s.get("y")
    ref_h, ref_x = layers.residual_norm(f64(s["h"]), None if y is None else f64(y), post, pre, eps, alpha,
                                        **vectors(s, "gate", "post_w", "pre_w", "scale", "shift"))
    for b in range(s["h"].shape[0]):
        for k, ref in (("h_out", ref_h), ("x", ref_x)):
            if k not in s:
                continue
            if b in skip:
                assert torch.isnan(s[k][b]).all()
                continue
            if ref[b].size == 0:
                continue
            mag = np.abs(ref[b]).max(-1, keepdims=True) + 1.0
            ok, worst = close(f64(s[k][b]), ref[b], mag)
            assert ok, (k, b, worst)


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
@pytest.mark.parametrize("C", [8, 264, 1152])
def test_residual_norm_kinds(cuda_ok, post, pre, C):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(100 * post + 10 * pre + C)
    segs = []
    for n, weights, wide in ((1, True, False), (37, False, True), (150, True, True)):
        s = norm_case(2, n, C, g, weights, wide)
        s["h_out"] = torch.full((2, n, C), float("nan"), dtype=torch.bfloat16, device="cuda")
        s["x"] = torch.full((2, n, C), float("nan"), dtype=torch.bfloat16, device="cuda")
        segs.append(s)
    api.refadapt_residual_norm(segs, C, post, pre, 1e-5, 0.75)
    torch.cuda.synchronize()
    for s in segs:
        check_forward(s, post, pre, 1e-5, 0.75)


@pytest.mark.parametrize("C,B,n", [(256, 70, 3), (512, 1, 4000), (2560, 2, 611), (3328, 1, 1), (4096, 5, 9),
                                   (5120, 1, 300), (4104, 2, 40)])
def test_residual_norm_sizes(cuda_ok, C, B, n):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(C + n)
    s = norm_case(B, n, C, g, True)
    s["h_out"], s["x"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
    api.refadapt_residual_norm([s], C, 2, 1)
    check_forward(s, 2, 1, 1e-6, 1.0)


def test_residual_norm_gated_segments_optional_parts_and_in_place(cuda_ok):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(3)
    B, C = 3, 640
    mode = torch.tensor([0, 2, 0], dtype=torch.int32, device="cuda")
    nan = float("nan")
    text, ref, tgt = norm_case(B, 20, C, g, False), norm_case(B, 90, C, g, True), norm_case(B, 33, C, g, True)
    for s in (text, ref, tgt):
        s["h_out"] = torch.full_like(s["h"], nan)
        s["x"] = torch.full_like(s["h"], nan)
    ref["gated"] = True
    del tgt["y"], tgt["h_out"], tgt["shift"]          # the first norm of a stack
    api.refadapt_residual_norm([text, ref, tgt], C, 2, 2, mode=mode)
    check_forward(text, 2, 2, 1e-6, 1.0)
    check_forward(ref, 2, 2, 1e-6, 1.0, skip=(0, 2))
    check_forward(tgt, 2, 2, 1e-6, 1.0)
    # the last of a stack has no next norm; in place
    last = norm_case(B, 50, C, g, True, mod=False)
    want = dict(last, h=last["h"].clone())
    last["h_out"] = last["h"]
    api.refadapt_residual_norm([last], C, 1, 0)
    check_forward(dict(want, h_out=last["h_out"]), 1, 0, 1e-6, 1.0)
    both = norm_case(B, 50, C, g, True)
    want = dict(both, h=both["h"].clone(), y=both["y"].clone())
    both["h_out"], both["x"] = both["h"], both["y"]
    api.refadapt_residual_norm([both], C, 0, 1)
    check_forward(dict(want, h_out=both["h_out"], x=both["x"]), 0, 1, 1e-6, 1.0)


def test_residual_norm_large_mean_and_zero_rows(cuda_ok):
    """A row far from zero keeps its variance; a constant row and a zero row
    divide by sqrt(eps); one NaN stays in its row."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(4)
    C = 1024
    h = torch.zeros((1, 6, C))
    h[0, 0] = 200.0 + torch.randn(C, generator=g)
    h[0, 1] = 3.0
    h[0, 3] = torch.randn(C, generator=g)
    h[0, 4] = torch.randn(C, generator=g) * 1e-18
    h[0, 5] = torch.randn(C, generator=g)
    h = h.to(torch.bfloat16).cuda()
    h[0, 5, 17] = float("nan")
    x = torch.empty_like(h)
    api.refadapt_residual_norm([{"h": h, "x": x}], C, 0, 1, 1e-6)
    hh = f64(h)
    ref = layers.residual_norm(hh[:, :5], None, 0, 1, 1e-6)[1]
    # at mean 200 and deviation 1 the fp32 mean is good to 2^-24 * 200 of the deviation: 1.2e-5
    ok, worst = close(f64(x)[:, :5], ref, 2.0 + 0 * ref)
    assert ok, worst
    assert torch.isnan(x[0, 5]).all()


GRADS = ("dh", "dy", "dgate", "dscale", "dshift", "dpost_w", "dpre_w")


def backward_case(s, n, C, B, drop=()):
    s = dict(s)
    e = torch.full((B, n, C), float("nan"), dtype=torch.bfloat16, device="cuda")
    s.update(dh=e.clone(), dy=e.clone())
    s.update({k: torch.full((B, C), float("nan"), device="cuda") for k in ("dgate", "dscale", "dshift")})
    s.update({k: torch.full((C,), float("nan"), device="cuda") for k in ("dpost_w", "dpre_w")})
    for k in drop:
        s.pop(k, None)
    return s


def check_backward(s, post, pre, eps, alpha, keep=None):
    src = keep or s
    h, y = f64(src["h"]), f64(src["y"]) if "y" in src else None
    dx = f64(src["dx"]) if "dx" in src else None
    dho = f64(src["dh_out"]) if "dh_out" in src else None
    vec = vectors(src, "gate", "post_w", "pre_w", "scale")
    ref = layers.residual_norm_grad(h, y, dx, dho, post, pre, eps, alpha, **vec)
    # sums of magnitudes of the terms of each column sum
    w, mod = (1.0 if vec["pre_w"] is None else np.abs(vec["pre_w"])), 1.0
    if vec["scale"] is not None:
        mod = np.abs(1.0 + vec["scale"][:, None, :])
    adx = 0.0 * h if dx is None else np.abs(dx)
    xh = np.abs(layers.normalise(pre, h, eps)[0])
    mags = {"dshift": adx.sum(1), "dscale": (adx * xh * w).sum(1), "dpre_w": (adx * xh * mod).sum((0, 1))}
    if y is not None:
        w, gt = (1.0 if vec["post_w"] is None else np.abs(vec["post_w"])), 1.0
        if vec["gate"] is not None:
            gt = np.abs(vec["gate"][:, None, :])
        t = np.abs(ref["dh"] / alpha) * np.abs(layers.normalise(post, y, eps)[0])
        # dH itself is a difference of terms as large as the largest of its row
        t = t + 2.0 ** -4 * np.abs(ref["dh"] / alpha).max(-1, keepdims=True)
        mags.update(dgate=(t * w).sum(1), dpost_w=(t * gt).sum((0, 1)))
    for k in GRADS:
        if k not in s:
            continue
        got = f64(s[k]) if s[k].dtype == torch.bfloat16 else d64(s[k])
        if got.size == 0:
            continue
        if k in ("dh", "dy"):
            ok, worst = close(got, ref[k], np.abs(ref[k]).max(-1, keepdims=True) + 1e-3)
            assert ok, (k, worst)
        else:
            err = np.abs(got - ref[k])
            assert (err <= 320 * 2.0 ** -24 * mags[k] + 1e-30).all(), (k, float((err / (mags[k] + 1e-30)).max()))


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
@pytest.mark.parametrize("B,n,C,wide", [(2, 37, 264, True), (1, 1, 8, False), (3, 205, 1152, False)])
def test_residual_norm_backward_kinds(cuda_ok, post, pre, B, n, C, wide):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(100 * post + 10 * pre + C)
    s = norm_case(B, n, C, g, True, wide)
    s["dx"], s["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case(s, n, C, B)
    ws = api.residual_norm_backward_workspace(B, n, C)
    api.refadapt_residual_norm_backward(s, C, post, pre, ws, 1e-5, 0.75)
    check_backward(s, post, pre, 1e-5, 0.75)


@pytest.mark.parametrize("C,B,n", [(256, 200, 3), (512, 1, 4000), (2560, 2, 611), (4096, 5, 9), (5120, 1, 300),
                                   (4104, 2, 40), (1024, 2, 0)])
def test_residual_norm_backward_sizes(cuda_ok, C, B, n):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(C + n)
    s = norm_case(B, n, C, g, True)
    s["dx"], s["dh_out"] = bf((B, n, C), g, 0.01), bf((B, n, C), g, 0.01)
    s = backward_case(s, n, C, B)
    ws = torch.full((api.refadapt_residual_norm_backward_workspace_size(B, n, C) // 4,), float("nan"), device="cuda")
    api.refadapt_residual_norm_backward(s, C, 2, 1, ws)
    check_backward(s, 2, 1, 1e-6, 1.0)
    first = {k: s[k].clone() for k in GRADS}
    api.refadapt_residual_norm_backward(s, C, 2, 1, ws)
    for k in GRADS:  # the same bits on every call
        assert torch.equal(s[k], first[k]), k


def test_residual_norm_backward_optional_parts_and_in_place(cuda_ok):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(8)
    B, n, C = 2, 90, 640
    ws = api.residual_norm_backward_workspace(B, n, C)
    full = norm_case(B, n, C, g, False, mod=False)
    full["dx"], full["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case({k: v for k, v in full.items() if k != "dx"}, n, C, B, ("dscale", "dpre_w"))
    api.refadapt_residual_norm_backward(s, C, 2, 1, ws)
    check_backward(s, 2, 1, 1e-6, 1.0)
    assert not s["dshift"].any()
    s = backward_case({k: v for k, v in full.items() if k not in ("dh_out", "y")}, n, C, B,
                      ("dy", "dgate", "dpost_w", "dshift"))
    api.refadapt_residual_norm_backward(s, C, 0, 1, ws)
    check_backward(s, 0, 1, 1e-6, 1.0)
    keep = {k: v.clone() for k, v in full.items()}
    s = backward_case(full, n, C, B, ("dgate", "dscale", "dshift", "dpost_w", "dpre_w"))
    s["dh"], s["dy"] = s["dh_out"], s["y"]
    api.refadapt_residual_norm_backward(s, C, 1, 2, ws)
    check_backward(s, 1, 2, 1e-6, 1.0, keep)


def test_residual_norm_refusals(cuda_ok):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RefAdaptError
    g = torch.Generator().manual_seed(1)
    s = norm_case(2, 6, 64, g, True)
    s["h_out"], s["x"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
    for bad, msg in (({"post": 3}, "known norms"), ({"eps": -1.0}, "eps"), ({"eps": math.nan}, "eps")):
        kw = dict({"post": 2, "pre": 1, "eps": 1e-6}, **bad)
        with pytest.raises(RefAdaptError, match=msg):
            api.refadapt_residual_norm([s], 64, kw["post"], kw["pre"], kw["eps"])
    with pytest.raises(RefAdaptError, match="gated but mode is NULL"):
        api.refadapt_residual_norm([dict(s, gated=True)], 64, 2, 1)
    with pytest.raises(RefAdaptError, match="both outputs"):
        api.refadapt_residual_norm([{"h": s["h"]}], 64, 2, 1)
    with pytest.raises(RefAdaptError, match="same tensor"):
        api.refadapt_residual_norm([dict(s, x=s["h_out"])], 64, 2, 1)
    with pytest.raises(RefAdaptError, match="sample stride"):
        api.refadapt_residual_norm([dict(s, x=s["x"][:1].expand(2, 6, 64))], 64, 2, 1)
    with pytest.raises(ValueError, match="y: expected"):
        api.refadapt_residual_norm([dict(s, y=s["y"][:, :5])], 64, 2, 1)
    with pytest.raises(ValueError, match="gate: expected"):
        api.refadapt_residual_norm([dict(s, gate=s["gate"][:1])], 64, 2, 1)
    with pytest.raises(ValueError, match="h: expected"):
        api.refadapt_residual_norm([dict(s, h=s["h"].float())], 64, 2, 1)
    big = torch.zeros((1, 1, 5128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RefAdaptError, match="5120"):
        api.refadapt_residual_norm([{"h": big, "x": big.clone()}], 5128, 0, 1)
    b = backward_case(dict(s, dx=s["h"], dh_out=s["h"]), 6, 64, 2, ("h_out", "x", "shift"))
    ws = api.residual_norm_backward_workspace(2, 6, 64)
    with pytest.raises(RefAdaptError, match="workspace"):
        api.refadapt_residual_norm_backward(b, 64, 2, 1, ws[:16])
    with pytest.raises(RefAdaptError, match="without y"):
        api.refadapt_residual_norm_backward({k: v for k, v in b.items() if k != "y"}, 64, 2, 1, ws)
    with pytest.raises(RefAdaptError, match="dx and dh_out"):
        api.refadapt_residual_norm_backward({k: v for k, v in b.items() if k not in ("dx", "dh_out")}, 64, 2, 1, ws)
    with pytest.raises(RefAdaptError, match="same tensor"):
        api.refadapt_residual_norm_backward(dict(b, dy=b["dh"]), 64, 2, 1, ws)


def test_residual_norm_backward_every_place_in_place(cuda_ok):
    """dh and dy in the place of any input, and refused where the strides differ."""
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RefAdaptError
    g = torch.Generator().manual_seed(12)
    B, n, C = 1, 70, 512
    ws = api.residual_norm_backward_workspace(B, n, C)
    for a, b in (("h", "dx"), ("dx", "dh_out"), ("y", "h"), ("dh_out", "y")):
        s = norm_case(B, n, C, g, True)
        s["dx"], s["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
        keep = {k: v.clone() for k, v in s.items()}
        s = backward_case(s, n, C, B)
        s["dh"], s["dy"] = s[a], s[b]
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        api.refadapt_residual_norm_backward(s, C, 2, 1, ws, err_word=err)
        api.refadapt_check_error(err)
        check_backward(s, 2, 1, 1e-6, 1.0, keep)
    s = norm_case(B, n, C, g, True)
    wide = bf((B, n, C + 64), g)
    s["h"], s["dx"], s["dh_out"] = wide[..., :C], bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case(s, n, C, B)
    s["dh"] = wide.reshape(-1)[:n * C].view(B, n, C)
    with pytest.raises(RefAdaptError, match="other strides"):
        api.refadapt_residual_norm_backward(s, C, 2, 1, ws)
