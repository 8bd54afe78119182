"""GPU parity of the gated feed-forward (refadapt_glu, refadapt_glu_backward)
against the fp64 oracle (oracle/layers.py) on the same inputs, and its refusals.

Tolerances. g and w are fp32 sums of C bf16 products in TMEM: off by at most a few
2^-24 times the sum of the products' magnitudes per term; with N(0, 1) operands
sum |t| is about 0.64 sqrt(C) of the result's deviation for weights of 1/sqrt(C),
so 2^-14 of the deviation has room. A bf16 output adds half a unit in the last
place, 2^-8 |ref|. Forward: |got - ref| <= 2^-8 |ref| (1 + 2^-5) + 2^-11 rms: the
product's relative error is that of both factors (their errors, against |g|, |w|
up to 4.5 deviations).
Gradients: dg and dw are rounded to bf16 as operands, a relative error of at most
2^-8 per term, independent between terms, so a sum of terms t is off by at most a
few 2^-8 / sqrt(3) * sqrt(sum t^2): six deviations of that, beside the output's own
rounding: |got - ref| <= 2^-8 |ref| (1 + 2^-5) + 6 * 2^-8 / sqrt(3) * sqrt(sum t^2)."""
import math

import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import layers

pytestmark = pytest.mark.gpu


def bf(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).cuda()


def wide(shape, g, scale=1.0):
    """Rows of a larger buffer: other row and sample strides."""
    B, n, F = shape
    return bf((B, n + 2, F + 24), g, scale)[:, 1:1 + n, 8:8 + F]


def forward_ok(got, ref):
    err = np.abs(f64(got) - ref)
    rms = math.sqrt(float((ref ** 2).mean())) if ref.size else 0.0
    tol = 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -5) + 2.0 ** -11 * rms
    return bool((err <= tol).all()), float((err / (tol + 1e-300)).max()) if ref.size else 0.0


def seg(B, n, C, F, g, save, strided=False):
    make = wide if strided else bf
    s = {"x": make((B, n, C), g), "w_gate": bf((F, C), g, C ** -0.5), "w_up": bf((F, C), g, C ** -0.5),
         "out": make((B, n, F), g)}
    s["out"].fill_(float("nan"))
    if save:
        s["pre_gate"], s["pre_up"] = torch.full_like(s["out"], float("nan")), make((B, n, F), g)
    return s


def check_forward(s, act, skip=()):
    u, g, w = layers.glu(f64(s["x"]), f64(s["w_gate"]), f64(s["w_up"]), act)
    for k, ref in (("out", u), ("pre_gate", g), ("pre_up", w)):
        if k not in s:
            continue
        for b in range(ref.shape[0]):
            if b in skip:
                assert torch.isnan(s[k][b]).all()
                continue
            ok, worst = forward_ok(s[k][b], ref[b])
            assert ok, (k, b, worst)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("rows,C,F", [(1, 64, 64), (1, 2048, 5504), (7, 520, 1000), (16, 1024, 2736), (17, 1024, 264),
                                      (33, 128, 4104), (77, 256, 72), (129, 1032, 648), (300, 712, 1368)])
def test_glu_rows_and_widths(cuda_ok, act, rows, C, F):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(rows + C + F)
    s = seg(1, rows, C, F, g, save=False)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.refadapt_glu([s], F, C, act, err_word=err)
    api.refadapt_check_error(err)
    check_forward(s, act)
    t = dict(s, pre_gate=torch.empty_like(s["out"]), pre_up=torch.empty_like(s["out"]), out=torch.empty_like(s["out"]))
    api.refadapt_glu([t], F, C, act, err_word=err)
    api.refadapt_check_error(err)
    check_forward(t, act)


@pytest.mark.parametrize("strided", [False, True])
def test_glu_segments_samples_and_modes(cuda_ok, strided):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(7)
    B, C, F = 3, 320, 808
    segs = [seg(B, 5, C, F, g, False, strided), seg(B, 140, C, F, g, True, strided), seg(B, 261, C, F, g, True, strided),
            ]
    segs[1]["gated"] = True
    segs[1]["out"].fill_(float("nan")), segs[1]["pre_up"].fill_(float("nan"))
    mode = torch.tensor([0, 3, 0], dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.refadapt_glu(segs, F, C, 0, mode=mode, err_word=err)
    api.refadapt_check_error(err)
    for i, s in enumerate(segs):
        check_forward(s, 0, skip=(0, 2) if i == 1 else ())
    # an empty segment beside others
    none = seg(B, 0, C, F, g, False)
    segs[0]["out"].fill_(float("nan"))
    api.refadapt_glu([none, segs[0]], F, C, 0)
    check_forward(segs[0], 0)


@pytest.mark.parametrize("rows", [3, 200])
def test_glu_extremes(cuda_ok, rows):
    """A gate far below zero gives zero, far above the product; NaN and infinity
    stay in their row."""
    from paper_2609_32415_gb300 import api
    C, F = 64, 128
    x = torch.zeros((1, rows, C))
    x[0, 0, 0], x[0, 1, 0], x[0, 2, 1] = 1.0, -1.0, float("nan")
    w_gate, w_up = torch.zeros((F, C)), torch.ones((F, C))
    w_gate[:, 0] = 300.0
    for act in (0, 1):
        s = {"x": x.to(torch.bfloat16).cuda(), "w_gate": w_gate.to(torch.bfloat16).cuda(),
             "w_up": w_up.to(torch.bfloat16).cuda(), "out": torch.empty((1, rows, F), dtype=torch.bfloat16, device="cuda")}
        api.refadapt_glu([s], F, C, act)
        out = f64(s["out"])[0]
        assert (out[0] == 300.0).all() and (out[1] == 0.0).all() and np.isnan(out[2]).all() and not out[3:].any()


def grads(B, n, C, F, O, g, act, strided=False):
    make = wide if strided else bf
    s = {"dy": make((B, n, O), g, 0.01), "x": make((B, n, C), g), "w_gate": bf((F, C), g, C ** -0.5),
         "w_up": bf((F, C), g, C ** -0.5), "w_down": bf((O, F), g, F ** -0.5)}
    u, gate, up = layers.glu(f64(s["x"]), f64(s["w_gate"]), f64(s["w_up"]), act)
    for k, v in (("pre_gate", gate), ("pre_up", up), ("hidden", u)):
        t = make((B, n, F), g)
        t.copy_(torch.from_numpy(v).to(torch.bfloat16))
        s[k] = t
    s["dx"] = make((B, n, C), g)
    s["dw_gate"], s["dw_up"], s["dw_down"] = (torch.full(sh, float("nan"), dtype=torch.bfloat16, device="cuda")
                                              for sh in ((F, C), (F, C), (O, F)))
    s["dx"].fill_(float("nan"))
    return s


def call(s, act, ws, err, drop=()):
    from paper_2609_32415_gb300 import api
    out = {k: s[k] for k in ("dx", "dw_gate", "dw_up", "dw_down") if k not in drop}
    api.refadapt_glu_backward(s["dy"], s.get("x"), s["w_gate"], s["w_up"], s["w_down"], s.get("pre_gate"),
                              s.get("pre_up"), s.get("hidden"), act, ws, err_word=err, **out)
    api.refadapt_check_error(err)


def check_grads(s, act, drop=()):
    flat = {k: f64(s[k]).reshape(-1, s[k].shape[-1]) for k in ("dy", "x", "pre_gate", "pre_up", "hidden")}
    w = {k: f64(s[k]) for k in ("w_gate", "w_up", "w_down")}
    ref = layers.glu_grad(flat["dy"], flat["x"], w["w_gate"], w["w_up"], w["w_down"], flat["pre_gate"], flat["pre_up"],
                          flat["hidden"], act)
    a, da = layers.activation(act, flat["pre_gate"])
    du = flat["dy"] @ w["w_down"]
    dg2, dw2 = (du * flat["pre_up"] * da) ** 2, (du * a) ** 2
    sq = {"dx": dg2 @ w["w_gate"] ** 2 + dw2 @ w["w_up"] ** 2, "dw_gate": dg2.T @ flat["x"] ** 2,
          "dw_up": dw2.T @ flat["x"] ** 2, "dw_down": (flat["dy"] ** 2).T @ flat["hidden"] ** 2}
    for k, r in ref.items():
        if k in drop or r.size == 0:
            continue
        got = f64(s[k]).reshape(r.shape)
        err = np.abs(got - r)
        tol = 2.0 ** -8 * np.abs(r) * (1 + 2.0 ** -5) + 6 * 2.0 ** -8 / math.sqrt(3) * np.sqrt(sq[k])
        assert (err <= tol).all(), (k, float((err / (tol + 1e-300)).max()))
        # dw_down has unrounded operands: its own rounding alone, and fp32 sums
        if k == "dw_down":
            assert (err <= 2.0 ** -8 * np.abs(r) * (1 + 2.0 ** -5) + 2.0 ** -14 * np.sqrt(sq[k])).all()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("B,n,C,F,O,strided", [
    (1, 1, 64, 64, 64, False), (1, 8, 512, 1024, 512, False), (1, 77, 520, 1000, 264, False),
    (2, 130, 256, 648, 256, True), (3, 64, 328, 200, 72, False), (1, 600, 256, 328, 256, False),
    (1, 2100, 64, 128, 136, True), (2, 33, 1024, 2736, 1024, False)])
def test_glu_backward(cuda_ok, act, B, n, C, F, O, strided):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(n + C + F)
    s = grads(B, n, C, F, O, g, act, strided)
    ws = torch.full((api.refadapt_glu_backward_workspace_size(B, n, C, F, O) // 2,), float("nan"), dtype=torch.bfloat16,
                    device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(s, act, ws, err)
    check_grads(s, act)
    first = {k: s[k].clone() for k in ("dx", "dw_gate", "dw_up", "dw_down")}
    call(s, act, ws, err)
    for k, v in first.items():  # the same bits on every call
        assert torch.equal(s[k], v), k


def test_glu_backward_wanted_gradients_only(cuda_ok):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(11)
    B, n, C, F, O = 1, 90, 128, 200, 128
    ws = api.glu_backward_workspace(B, n, C, F, O)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    every = ("dx", "dw_gate", "dw_up", "dw_down")
    for want, absent in ((("dx",), ("x", "hidden")), (("dw_up",), ("hidden",)), (("dw_down",), ("x", "pre_gate", "pre_up")),
                         (("dx", "dw_gate"), ("hidden",))):
        s = grads(B, n, C, F, O, g, 0)
        drop = [k for k in every if k not in want]
        call({k: v for k, v in s.items() if k not in absent}, 0, ws, err, drop)
        check_grads(s, 0, drop)
        for k in drop:
            assert torch.isnan(s[k]).all(), k
    s = grads(B, 0, C, F, O, g, 0)
    call(s, 0, api.glu_backward_workspace(B, 0, C, F, O), err)
    for k in ("dw_gate", "dw_up", "dw_down"):
        assert not s[k].any()


def test_glu_backward_matches_differences_of_the_forward_call(cuda_ok):
    """Directional differences of the forward kernels' own loss. With steps of
    2^-3 in bf16-exact inputs the second-order term cancels in the central
    difference; what is left is the outputs' rounding, 2^-9 per element of sums
    that add up as a random walk, and the third derivative."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(21)
    B, n, C, F, O = 1, 64, 128, 256, 128
    s = grads(B, n, C, F, O, g, 0)
    v = (torch.randint(0, 2, (B, n, C), generator=g).float() * 2 - 1).cuda()
    x = (s["x"].float() * 8).round() / 8
    s["x"] = x.to(torch.bfloat16)
    dy = s["dy"].float()

    def loss(h):
        t = {"x": (x + h * v).to(torch.bfloat16), "w_gate": s["w_gate"], "w_up": s["w_up"], "out": s["hidden"].clone()}
        api.refadapt_glu([t], F, C, 0)
        return float((t["out"].double() @ s["w_down"].double().T * dy.double()).sum())

    t = {"x": s["x"], "w_gate": s["w_gate"], "w_up": s["w_up"], "out": s["hidden"], "pre_gate": s["pre_gate"],
         "pre_up": s["pre_up"]}
    api.refadapt_glu([t], F, C, 0)
    call(s, 0, api.glu_backward_workspace(B, n, C, F, O), torch.zeros(1, dtype=torch.int32, device="cuda"))
    h = 2.0 ** -3
    got = float((s["dx"].double() * v.double()).sum())
    want = (loss(h) - loss(-h)) / (2 * h)
    # rounding of `hidden`: 2^-9 |hidden| per element, through w_down and dy, over 2 h
    du = (dy.double() @ s["w_down"].double()).abs()
    noise = 6 * 2.0 ** -9 / math.sqrt(3) * float(((du * s["hidden"].double()) ** 2).sum().sqrt()) * math.sqrt(2) / (2 * h)
    third = 2.0 ** -4 * float((s["dx"].double() ** 2).sum().sqrt())  # h^2 / 6 of a third derivative up to 24 times the first
    assert abs(got - want) <= noise + third, (got, want, noise, third)


def test_glu_refusals(cuda_ok):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RefAdaptError
    g = torch.Generator().manual_seed(1)
    s = seg(2, 6, 64, 128, g, True)
    with pytest.raises(RefAdaptError, match="known activation"):
        api.refadapt_glu([s], 128, 64, 2)
    with pytest.raises(RefAdaptError, match="gated but mode is NULL"):
        api.refadapt_glu([dict(s, gated=True)], 128, 64, 0)
    with pytest.raises(RefAdaptError, match="go together"):
        api.refadapt_glu([dict(s, pre_up=None)], 128, 64, 0)
    with pytest.raises(ValueError, match="w_up: expected"):
        api.refadapt_glu([dict(s, w_up=s["w_up"][:, :56])], 128, 64, 0)
    with pytest.raises(ValueError, match="out: expected"):
        api.refadapt_glu([dict(s, out=s["out"][:, :5])], 128, 64, 0)
    with pytest.raises(ValueError, match="x: expected"):
        api.refadapt_glu([dict(s, x=s["x"].half())], 128, 64, 0)
    small = seg(1, 6, 56, 128, g, False)
    with pytest.raises(RefAdaptError, match="at least 64"):
        api.refadapt_glu([small], 128, 56, 0)
    odd = torch.zeros((2, 6, 72), dtype=torch.bfloat16, device="cuda")[..., 1:65]
    with pytest.raises(RefAdaptError, match="aligned"):
        api.refadapt_glu([dict(s, x=odd)], 128, 64, 0)
    with pytest.raises(TypeError):
        api.refadapt_glu([], 128, 64, 0)
    b = grads(1, 6, 64, 128, 72, g, 0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = api.glu_backward_workspace(1, 6, 64, 128, 72)
    with pytest.raises(RefAdaptError, match="workspace"):
        call(b, 0, ws[:64], err)
    with pytest.raises(RefAdaptError, match="no gradient"):
        call(b, 0, ws, err, ("dx", "dw_gate", "dw_up", "dw_down"))
    with pytest.raises(RefAdaptError, match="x must be given"):
        call({k: v for k, v in b.items() if k != "x"}, 0, ws, err)
    with pytest.raises(RefAdaptError, match="hidden must be given"):
        call({k: v for k, v in b.items() if k != "hidden"}, 0, ws, err)
    with pytest.raises(ValueError, match="dw_down: expected"):
        call(dict(b, dw_down=b["dw_down"].float()), 0, ws, err)


def test_glu_overlapping_outputs_are_refused(cuda_ok):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RefAdaptError
    g = torch.Generator().manual_seed(2)
    s = seg(1, 40, 128, 128, g, True)
    for bad in ({"out": s["x"]}, {"pre_up": s["pre_gate"]}, {"pre_gate": s["out"]}):
        with pytest.raises(RefAdaptError, match="overlap"):
            api.refadapt_glu([dict(s, **bad)], 128, 128, 0)
    b = grads(1, 40, 128, 128, 128, g, 0)
    ws = api.glu_backward_workspace(1, 40, 128, 128, 128)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for k in ("dy", "x", "hidden"):
        with pytest.raises(RefAdaptError, match="overlap"):
            call(dict(b, dx=b[k]), 0, ws, err)


def test_glu_many_tiles(cuda_ok):
    """More tile rows than a band, several bands, and a last band that is not full."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(31)
    s = seg(1, 256 * 35 + 9, 64, 264, g, False)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.refadapt_glu([s], 264, 64, 0, err_word=err)
    api.refadapt_check_error(err)
    check_forward(s, 0)
    s = grads(2, 256 * 17 + 100, 64, 520, 64, g, 1)
    call(s, 1, api.glu_backward_workspace(2, 256 * 17 + 100, 64, 520, 64), err)
    check_grads(s, 1)
