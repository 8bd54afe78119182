"""The residual norm's column sums (dgate, dscale, dshift, dpost_w, dpre_w) over long runs
of rows, all of them against 64 bits: a row that a slot's reuse skipped or counted twice, a
wrong group or a wrong share shows here.

Bound. A sum's longest chain of fp32 additions: the rows of a CTA (B n / 100 at most: a call
of this size is cut for more CTAs than that), its groups (10), the shares of 32 warps (5),
the 32 of them, the samples; with a term's own roundings (16 half units) that is
(B n / 100 + 80) 2^-24 of the terms' magnitudes, where a term of dgate and dpost_w is a
difference of parts as large as its row's largest (a sixteenth of that counted in). An
average row's term is 1 / (B n) of the magnitudes, ten times that bound at 9000 rows."""
import math

import pytest
import torch

from test_gpu_block_layers import backward_case, bf, norm_case

pytestmark = pytest.mark.gpu


def normalised(kind, v, eps=1e-6):
    if kind == 0:
        return v, torch.ones_like(v[..., :1])
    c = v - v.mean(-1, keepdim=True) if kind == 1 else v
    r = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    return c * r, r


def reference(s, post, pre):
    """{name: (sums, sums of the terms' magnitudes)} in 64 bits on the GPU."""
    d = {k: s[k].double() for k in ("h", "y", "dx", "dh_out", "gate", "scale", "post_w", "pre_w")}
    gate, mod = d["gate"][:, None], 1.0 + d["scale"][:, None]
    xh, r = normalised(pre, d["h"])
    e = d["dx"] * d["pre_w"] * mod
    if pre == 1:
        e = e - e.mean(-1, keepdim=True)
    if pre != 0:
        e = r * (e - xh * (d["dx"] * d["pre_w"] * mod * xh).mean(-1, keepdim=True))
    dH = d["dh_out"] + e
    yh, _ = normalised(post, d["y"])
    t0, t1, t2 = d["dx"], d["dx"] * xh, dH * yh
    m2 = t2.abs() + 2.0 ** -4 * dH.abs().amax(-1, keepdim=True)

    def sums(t, m, per_sample, weights):
        f = weights.expand_as(t)
        return ((t * per_sample).sum(1), (m * per_sample.abs()).sum(1)) if per_sample is not None else \
            ((t * f).sum((0, 1)), (m * f.abs()).sum((0, 1)))

    one = torch.ones_like(d["pre_w"])
    return {"dshift": sums(t0, t0.abs(), one, one), "dscale": sums(t1, t1.abs(), d["pre_w"], one),
            "dgate": sums(t2, m2, d["post_w"], one), "dpre_w": sums(t1, t1.abs(), None, mod),
            "dpost_w": sums(t2, m2, None, gate)}


@pytest.mark.parametrize("post,pre", [(0, 0), (0, 1), (1, 2), (1, 1), (2, 2)])
@pytest.mark.parametrize("C,B,n", [(200, 1, 9001), (504, 2, 4500), (640, 1, 9000), (768, 1, 9000), (1160, 1, 6100),
                                   (2560, 1, 4700), (5120, 2, 1501)])
def test_column_sums_of_long_runs(cuda_ok, C, B, n, post, pre):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(C + n + 10 * post + pre)
    s = norm_case(B, n, C, g, True)
    s["dx"], s["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case(s, n, C, B)
    api.refadapt_residual_norm_backward(s, C, post, pre, api.residual_norm_backward_workspace(B, n, C))
    bound = (math.ceil(B * n / 100) + 80) * 2.0 ** -24
    for k, (want, mag) in reference(s, post, pre).items():
        worst = float(((s[k].double() - want).abs() / mag).max())
        assert worst <= bound, (k, worst, bound)
