"""Timed cases of the operators of a DiT block around the joint attention: the gated
feed-forward block, the norms before and after a branch with its gate and residual
scale, and rotary positions with several axes; each with its backward pass.

Kinds:

  glu        refadapt_glu: u = act(x Wg^T) o (x Wu^T), one or two streams in a call
             (text rows with their weights, image rows with theirs), with the
             pre-activations kept for training where `save` is true;
  glu_grad   refadapt_glu_backward: the gradients of y = u Wd^T with respect to x and the
             three weights, from dy and what the forward call kept;
  norm       refadapt_residual_norm: h' = alpha h + gate o N_post(y) w_post, then
             x = N_pre(h') w_pre (1 + scale) + shift;
  norm_grad  refadapt_residual_norm_backward: the gradients of h, y, gate, scale, shift
             and of the norms' weights;
  rope       refadapt_rope_axes on q and k (inverse: the backward pass).

Values: rows that enter a projection are N(0, 1) (they come out of a norm), weights
N(0, 1) / sqrt(fan_in), gradients 0.01 N(0, 1); AdaLN scale and shift 0.1 N(0, 1), gates
0.3 + 0.05 N(0, 1), norm weights 1 + 0.1 N(0, 1); q and k N(0, 1); positions are the
grid coordinates of a text, image or video token, centred in height and width.
"""
import math

import torch

own = False

MAX_FLOPS = 9.0e11   # of the largest listed call
MAX_BYTES = 4.1e8
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
NORMS = {"none": NORM_NONE, "layer": NORM_LAYER, "rms": NORM_RMS}
ACTS = {"silu": 0, "gelu": 1}
EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # One row through the gated projections: a pooled or conditioning token, alone
        # in its call. Latency and the weights' bytes.
        dict(name="glu_single_row", kind="glu", B=1, text=1, image=0, C=2048, F=5504, act="silu", save=False),
        # A draft of two samples, ragged text and image rows, a width that is not a
        # multiple of a tile.
        dict(name="glu_draft", kind="glu", B=2, text=77, image=500, C=1024, F=2736, act="gelu", save=False),
        # The rows of an image-edit block that reuses (text and target rows).
        dict(name="glu_image", kind="glu", B=1, text=256, image=4096, C=2048, F=8192, act="silu", save=False),
        # Training on a few ragged rows of a small model.
        dict(name="glu_grad_draft", kind="glu_grad", B=1, rows=377, C=1024, F=2736, act="gelu"),
        # Training on an image's rows: the largest call.
        dict(name="glu_grad_image", kind="glu_grad", B=1, rows=4333, C=2048, F=8192, act="silu"),
        # One row between two branches: latency.
        dict(name="norm_single_row", kind="norm", B=1, text=1, image=0, C=2048, post="rms", pre="rms", weights=True),
        # Text and image rows of two samples between attention and feed-forward.
        dict(name="norm_image", kind="norm", B=2, text=256, image=4096, C=2560, post="rms", pre="layer",
             weights=False),
        # Training, a small ragged draft of three samples, both norms with weights.
        dict(name="norm_grad_draft", kind="norm_grad", B=3, rows=205, C=1152, post="layer", pre="rms", weights=True),
        # Training on two images' rows.
        dict(name="norm_grad_image", kind="norm_grad", B=2, rows=4096, C=2560, post="rms", pre="layer", weights=True),
        # One token's heads: latency.
        dict(name="rope_single_token", kind="rope", B=1, frames=1, height=1, width=1, H=16, Hk=16, d=128,
             axes="16,56,56", tokens=True, inverse=False),
        # A video clip's q and k: frames x height x width, head-major.
        dict(name="rope_video", kind="rope", B=1, frames=16, height=24, width=42, H=24, Hk=24, d=128, axes="16,56,56",
             tokens=False, inverse=False),
        # The backward pass of two images' q and shared k heads, token-major.
        dict(name="rope_grad_image", kind="rope", B=2, frames=1, height=45, width=61, H=16, Hk=4, d=64, axes="8,28,28",
             tokens=True, inverse=True),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rows(rng, lo, hi):
    """A row count between lo and hi, odd ones and multiples of 128 among them."""
    n = _log(rng, lo, hi)
    return n // 128 * 128 if n >= 256 and rng.random() < 0.3 else n


def _draw(rng):
    kind = rng.choice(["glu", "glu", "glu_grad", "norm", "norm_grad", "rope"])
    if kind == "glu":
        C = 8 * _log(rng, 64, 512)
        return dict(kind=kind, B=rng.choice([1, 1, 2]), text=_rows(rng, 1, 512),
                    image=rng.choice([0, _rows(rng, 16, 8192)]), C=C, F=8 * _log(rng, 128, 1376),
                    act=rng.choice(list(ACTS)), save=rng.random() < 0.4)
    if kind == "glu_grad":
        return dict(kind=kind, B=rng.choice([1, 1, 2]), rows=_rows(rng, 8, 8192), C=8 * _log(rng, 64, 384),
                    F=8 * _log(rng, 128, 1376), act=rng.choice(list(ACTS)))
    if kind == "norm":
        return dict(kind=kind, B=rng.choice([1, 2, 3]), text=_rows(rng, 1, 512),
                    image=rng.choice([0, _rows(rng, 16, 16384)]), C=8 * _log(rng, 32, 640),
                    post=rng.choice(list(NORMS)), pre=rng.choice(["layer", "rms"]), weights=rng.random() < 0.5)
    if kind == "norm_grad":
        return dict(kind=kind, B=rng.choice([1, 2, 3]), rows=_rows(rng, 1, 16384), C=8 * _log(rng, 32, 640),
                    post=rng.choice(list(NORMS)), pre=rng.choice(["layer", "rms"]), weights=rng.random() < 0.5)
    d, axes = rng.choice([(64, "8,28,28"), (64, "32,32"), (128, "16,56,56"), (128, "44,44,40"), (96, "32,32,32")])
    H = rng.choice([8, 16, 24, 32])
    return dict(kind=kind, B=rng.choice([1, 1, 2]), frames=rng.choice([1, 1, rng.randint(2, 21)]),
                height=_log(rng, 1, 64), width=_log(rng, 1, 64), H=H, Hk=rng.choice([H, H // 4]), d=d, axes=axes,
                tokens=rng.random() < 0.5, inverse=rng.random() < 0.4)


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return case


# ------------------------------------------------------------------ inputs
def _streams(case):
    return [case[r] for r in ("text", "image") if case[r] > 0]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(dtype)

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    f32 = torch.float32
    st = {"case": case, "B": case["B"]}
    if case["kind"] in ("glu", "glu_grad"):
        B, C, F = case["B"], case["C"], case["F"]
        st["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if case["kind"] == "glu":
            st["segs"] = []
            for n in _streams(case):
                s = {"x": normal(B, n, C), "w_gate": normal(F, C, scale=C ** -0.5),
                     "w_up": normal(F, C, scale=C ** -0.5), "out": empty(B, n, F)}
                if case["save"]:
                    s["pre_gate"], s["pre_up"] = empty(B, n, F), empty(B, n, F)
                st["segs"].append(s)
            return st
        n = case["rows"]
        st["dy"], st["x"] = normal(B, n, C, scale=0.01), normal(B, n, C)
        st["w_gate"], st["w_up"] = normal(F, C, scale=C ** -0.5), normal(F, C, scale=C ** -0.5)
        st["w_down"] = normal(C, F, scale=F ** -0.5)
        # what the forward call keeps
        st["pre_gate"] = st["x"] @ st["w_gate"].T
        st["pre_up"] = st["x"] @ st["w_up"].T
        st["hidden"] = (_act(case["act"], st["pre_gate"].float()) * st["pre_up"].float()).to(torch.bfloat16)
        st["dx"] = empty(B, n, C)
        st["dw_gate"], st["dw_up"], st["dw_down"] = empty(F, C), empty(F, C), empty(C, F)
        return st
    if case["kind"] in ("norm", "norm_grad"):
        B, C = case["B"], case["C"]
        train = case["kind"] == "norm_grad"
        st["segs"] = []
        for n in [case["rows"]] if train else _streams(case):
            s = {"h": normal(B, n, C, scale=2.0), "y": normal(B, n, C, scale=1.5, mean=0.1),
                 "gate": normal(B, C, scale=0.05, mean=0.3, dtype=f32), "scale": normal(B, C, scale=0.1, dtype=f32),
                 "shift": normal(B, C, scale=0.1, dtype=f32)}
            if case["weights"]:
                s["pre_w"] = normal(C, scale=0.1, mean=1.0, dtype=f32)
                if case["post"] != "none":
                    s["post_w"] = normal(C, scale=0.1, mean=1.0, dtype=f32)
            if train:
                s["dx"], s["dh_out"] = normal(B, n, C, scale=0.01), normal(B, n, C, scale=0.01)
                s["dh"], s["dy"] = empty(B, n, C), empty(B, n, C)
                s.update({k: empty(B, C, dtype=f32) for k in ("dgate", "dscale", "dshift")})
                s.update({"d" + k: empty(C, dtype=f32) for k in ("pre_w", "post_w") if k in s})
            else:
                s["h_out"], s["x"] = empty(B, n, C), empty(B, n, C)
            st["segs"].append(s)
        st["alpha"] = 1.0
        return st
    B, d, axes = case["B"], case["d"], [int(a) for a in case["axes"].split(",")]
    t, hh, ww = case["frames"], case["height"], case["width"]
    n = t * hh * ww
    grid = torch.stack(torch.meshgrid(torch.arange(t, device="cuda", dtype=f32),
                                      torch.arange(hh, device="cuda", dtype=f32) - hh // 2,
                                      torch.arange(ww, device="cuda", dtype=f32) - ww // 2, indexing="ij"), -1)
    # the samples of a batch differ in the offset of their first frame, as references and targets do
    off = torch.randint(0, 64, (B, 1, 1), generator=g, device="cuda").to(f32)
    pos = grid.reshape(1, n, 3).repeat(B, 1, 1)
    pos[:, :, :1] += off
    st["pos"] = pos[..., 3 - len(axes):].contiguous()
    st["axes"] = axes

    def heads(H):
        if case["tokens"]:
            return normal(B, n, H, d).permute(0, 2, 1, 3), empty(B, n, H, d).permute(0, 2, 1, 3)
        return normal(B, H, n, d), empty(B, H, n, d)

    st["q"], st["q_out"] = heads(case["H"])
    st["k"], st["k_out"] = heads(case["Hk"])
    return st


# ------------------------------------------------------------------ plain forms
def _act(act, g):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def _act_grad(act, g):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _bf(x):
    return x.to(torch.bfloat16)


def _plain_glu(case, s):
    x = s["x"].float()
    g, w = x @ s["w_gate"].float().T, x @ s["w_up"].float().T
    out = {"out": _bf(_act(case["act"], g) * w)}
    if case["save"]:
        out.update(pre_gate=_bf(g), pre_up=_bf(w))
    return out


def _plain_glu_grad(case, st):
    flat = {k: st[k].float().reshape(-1, st[k].shape[-1]) for k in ("dy", "x", "pre_gate", "pre_up", "hidden")}
    du = flat["dy"] @ st["w_down"].float()
    dg = du * flat["pre_up"] * _act_grad(case["act"], flat["pre_gate"])
    dw = du * _act(case["act"], flat["pre_gate"])
    dx = dg @ st["w_gate"].float() + dw @ st["w_up"].float()
    return {"dx": _bf(dx).reshape(st["x"].shape), "dw_gate": _bf(dg.T @ flat["x"]), "dw_up": _bf(dw.T @ flat["x"]),
            "dw_down": _bf(flat["dy"].T @ flat["hidden"])}


def _norm(kind, v):
    """Normalised rows and 1 / deviation."""
    if kind == "none":
        return v, 1.0
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _norm_grad(kind, vh, r, e):
    if kind == "none":
        return e
    if kind == "layer":
        e = e - e.mean(-1, keepdim=True)
    return r * (e - vh * (e * vh).mean(-1, keepdim=True))


def _plain_norm(case, st, s):
    z = _norm(case["post"], s["y"].float())[0] * s.get("post_w", 1.0)
    h = st["alpha"] * s["h"].float() + s["gate"][:, None] * z
    x = _norm(case["pre"], h)[0] * s.get("pre_w", 1.0) * (1 + s["scale"][:, None]) + s["shift"][:, None]
    return {"h_out": _bf(h), "x": _bf(x)}


def _plain_norm_grad(case, st, s):
    pre_w, post_w = s.get("pre_w", 1.0), s.get("post_w", 1.0)
    dx, mod, gate = s["dx"].float(), 1 + s["scale"][:, None], s["gate"][:, None]
    xh, r = _norm(case["pre"], s["h"].float())
    dh = s["dh_out"].float() + _norm_grad(case["pre"], xh, r, dx * pre_w * mod)
    zh, rz = _norm(case["post"], s["y"].float())
    dy = _norm_grad(case["post"], zh, rz, dh * gate * post_w)
    out = {"dh": _bf(st["alpha"] * dh), "dy": _bf(dy), "dshift": dx.sum(1), "dscale": (dx * xh * pre_w).sum(1),
           "dgate": (dh * zh * post_w).sum(1)}
    if "pre_w" in s:
        out["dpre_w"] = (dx * xh * mod).sum((0, 1))
    if "post_w" in s:
        out["dpost_w"] = (dh * zh * gate).sum((0, 1))
    return out


def _plain_rope(case, st, v):
    axes = st["axes"]
    ang = torch.cat([st["pos"][..., a:a + 1] *
                     BASE ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float32) / D)
                     for a, D in enumerate(axes)], -1)[:, None]
    c, s = torch.cos(ang), torch.sin(ang) * (-1.0 if case["inverse"] else 1.0)
    e, o = v.float()[..., 0::2], v.float()[..., 1::2]
    return _bf(torch.stack((e * c - o * s, e * s + o * c), -1).flatten(-2))


def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["kind"] == "glu":
        return [_plain_glu(case, s) for s in state["segs"]]
    if case["kind"] == "glu_grad":
        return _plain_glu_grad(case, state)
    if case["kind"] == "norm":
        return [_plain_norm(case, state, s) for s in state["segs"]]
    if case["kind"] == "norm_grad":
        return _plain_norm_grad(case, state, state["segs"][0])
    return {"q": _plain_rope(case, state, state["q"]), "k": _plain_rope(case, state, state["k"])}


def _run_own(case, st):
    from paper_2609_32415_gb300 import api

    if case["kind"] == "glu":
        api.refadapt_glu(st["segs"], case["F"], case["C"], ACTS[case["act"]], err_word=st["err"])
        return [{k: s[k] for k in ("out", "pre_gate", "pre_up") if k in s} for s in st["segs"]]
    if case["kind"] == "glu_grad":
        if "ws" not in st:
            st["ws"] = api.glu_backward_workspace(st["B"], case["rows"], case["C"], case["F"], case["C"])
        api.refadapt_glu_backward(st["dy"], st["x"], st["w_gate"], st["w_up"], st["w_down"], st["pre_gate"],
                                  st["pre_up"], st["hidden"], ACTS[case["act"]], st["ws"], dx=st["dx"],
                                  dw_gate=st["dw_gate"], dw_up=st["dw_up"], dw_down=st["dw_down"], err_word=st["err"])
        return {k: st[k] for k in ("dx", "dw_gate", "dw_up", "dw_down")}
    if case["kind"] == "norm":
        api.refadapt_residual_norm(st["segs"], case["C"], NORMS[case["post"]], NORMS[case["pre"]], EPS, st["alpha"])
        return [{"h_out": s["h_out"], "x": s["x"]} for s in st["segs"]]
    if case["kind"] == "norm_grad":
        s = st["segs"][0]
        if "ws" not in st:
            st["ws"] = api.residual_norm_backward_workspace(st["B"], case["rows"], case["C"])
        api.refadapt_residual_norm_backward(s, case["C"], NORMS[case["post"]], NORMS[case["pre"]], st["ws"], EPS,
                                            st["alpha"])
        return {k: s[k] for k in ("dh", "dy", "dshift", "dscale", "dgate", "dpre_w", "dpost_w") if k in s}
    api.refadapt_rope_axes([(st["q"], st["q_out"]), (st["k"], st["k_out"])], st["pos"], st["axes"], BASE,
                           inverse=case["inverse"])
    return {"q": st["q_out"], "k": st["k_out"]}


# ------------------------------------------------------------------ what a call cannot do without
def work(case):
    if case["kind"] == "glu":
        B, C, F = case["B"], case["C"], case["F"]
        R = B * sum(_streams(case))
        return {"bytes": 2.0 * R * C + 4.0 * F * C * len(_streams(case)) + (6.0 if case["save"] else 2.0) * R * F,
                "flops": 4.0 * R * C * F}
    if case["kind"] == "glu_grad":
        C, F, R = case["C"], case["F"], case["B"] * case["rows"]
        return {"bytes": 2.0 * R * (3 * C + 3 * F) + 12.0 * F * C, "flops": 12.0 * R * C * F}
    if case["kind"] == "norm":
        B, C, streams = case["B"], case["C"], _streams(case)
        vec = 12.0 * B * C + (4.0 * C * (2 if case["post"] != "none" else 1) if case["weights"] else 0.0)
        return {"bytes": 8.0 * B * sum(streams) * C + vec * len(streams), "flops": 20.0 * B * sum(streams) * C}
    if case["kind"] == "norm_grad":
        B, C, n = case["B"], case["C"], case["rows"]
        vec = 20.0 * B * C + (8.0 * C * (2 if case["post"] != "none" else 1) if case["weights"] else 0.0)
        return {"bytes": 12.0 * B * n * C + vec, "flops": 40.0 * B * n * C}
    B, n = case["B"], case["frames"] * case["height"] * case["width"]
    elems = float(B * n * (case["H"] + case["Hk"]) * case["d"])
    return {"bytes": 4.0 * elems + 4.0 * B * n * len(case["axes"].split(",")), "flops": 3.0 * elems}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The same results from their definitions in 64 bits; gradients through autograd."""
    st = prepare(case, seed)

    def wide(t):
        return t.double().requires_grad_(True)

    def activation(g):
        if case["act"] == "silu":
            return g * torch.sigmoid(g)
        return torch.nn.functional.gelu(g, approximate="tanh")

    def normalise(kind, v):
        if kind == "none":
            return v
        m = v.mean(-1, keepdim=True) if kind == "layer" else 0.0
        var = ((v - m) ** 2).mean(-1, keepdim=True)
        return (v - m) / torch.sqrt(var + EPS)

    if case["kind"] == "glu":
        res = []
        for s in st["segs"]:
            g = torch.einsum("bnc,fc->bnf", s["x"].double(), s["w_gate"].double())
            w = torch.einsum("bnc,fc->bnf", s["x"].double(), s["w_up"].double())
            res.append({"out": activation(g) * w, **({"pre_gate": g, "pre_up": w} if case["save"] else {})})
        return res
    if case["kind"] == "glu_grad":
        # the product's gradients at the kept pre-activations, then those of the three linear layers
        dy, x = st["dy"].double().flatten(0, 1), st["x"].double().flatten(0, 1)
        g, w = wide(st["pre_gate"].flatten(0, 1)), wide(st["pre_up"].flatten(0, 1))
        u = activation(g) * w
        u.backward(dy @ st["w_down"].double())
        dx = g.grad @ st["w_gate"].double()
        dx += w.grad @ st["w_up"].double()
        return {"dx": dx.reshape(st["x"].shape), "dw_gate": g.grad.T @ x, "dw_up": w.grad.T @ x,
                "dw_down": dy.T @ st["hidden"].double().flatten(0, 1)}
    if case["kind"] == "norm":
        res = []
        for s in st["segs"]:
            z = normalise(case["post"], s["y"].double())
            if "post_w" in s:
                z = z * s["post_w"].double()
            h = st["alpha"] * s["h"].double() + s["gate"].double()[:, None, :] * z
            x = normalise(case["pre"], h)
            if "pre_w" in s:
                x = x * s["pre_w"].double()
            res.append({"h_out": h, "x": x * (1 + s["scale"].double()[:, None, :]) + s["shift"].double()[:, None, :]})
        return res
    if case["kind"] == "norm_grad":
        # h holds the forward call's h': x is a function of it, and it of h and y
        s = st["segs"][0]
        y, gate, scale, shift = wide(s["y"]), wide(s["gate"]), wide(s["scale"]), wide(s["shift"])
        pre_w = wide(s["pre_w"]) if "pre_w" in s else torch.ones((), dtype=torch.float64, device="cuda")
        post_w = wide(s["post_w"]) if "post_w" in s else torch.ones((), dtype=torch.float64, device="cuda")
        h = wide(s["h"])
        x = normalise(case["pre"], h) * pre_w * (1 + scale[:, None, :]) + shift[:, None, :]
        x.backward(s["dx"].double())
        total = s["dh_out"].double() + h.grad
        branch = gate[:, None, :] * (normalise(case["post"], y) * post_w)
        branch.backward(total)
        out = {"dh": st["alpha"] * total, "dy": y.grad, "dshift": shift.grad, "dscale": scale.grad, "dgate": gate.grad}
        out.update({"d" + k: v.grad for k, v in (("pre_w", pre_w), ("post_w", post_w)) if k in s})
        return out
    axes = [int(a) for a in case["axes"].split(",")]
    col = torch.tensor([a for a, D in enumerate(axes) for _ in range(D // 2)], device="cuda")
    freq = torch.tensor([BASE ** (-2.0 * i / D) for D in axes for i in range(D // 2)], dtype=torch.float64,
                        device="cuda")
    ang = st["pos"].double()[..., col] * freq
    turn = torch.polar(torch.ones_like(ang), -ang if case["inverse"] else ang)[:, None]

    def rotate(v):
        return torch.view_as_real(torch.view_as_complex(v.double().reshape(*v.shape[:-1], -1, 2)) * turn).flatten(-2)

    return {"q": rotate(st["q"]), "k": rotate(st["k"])}
