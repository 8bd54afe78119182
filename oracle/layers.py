"""fp64 oracle of the layers of gated DiT blocks: rotary positions with several
axes, norms before and after a branch, the gated feed-forward; their gradients.

Plain numpy from the definitions, without the package's code. Arrays are
float64; a row's features are the last axis."""
import numpy as np

NONE, LAYER, RMS = 0, 1, 2
SILU, GELU = 0, 1


# ------------------------------------------------------------------ rotary positions
def rope_axes_angles(pos, axes, base=10000.0):
    """[..., n_axes] coordinates -> [..., sum(axes) / 2] angles."""
    pos = np.asarray(pos, np.float64)
    return np.concatenate([pos[..., a:a + 1] * base ** (-np.arange(0, D, 2) / D) for a, D in enumerate(axes)], -1)


def rope_axes(x, pos, axes, base=10000.0, inverse=False):
    """x [B, H, n, d], pos [n, n_axes] or [B, n, n_axes]."""
    ang = rope_axes_angles(pos, axes, base)
    ang = ang[None, None] if ang.ndim == 2 else ang[:, None]
    c, s = np.cos(ang), np.sin(ang) * (-1.0 if inverse else 1.0)
    m = 2 * ang.shape[-1]
    out = np.array(x, np.float64)
    e, o = x[..., 0:m:2], x[..., 1:m:2]
    out[..., 0:m:2] = e * c - o * s
    out[..., 1:m:2] = e * s + o * c
    return out


# ------------------------------------------------------------------ norms around a branch
def normalise(kind, v, eps):
    """(normalised rows, 1 / deviation)."""
    if kind == NONE:
        return v, np.ones(v.shape[:-1] + (1,))
    c = v - v.mean(-1, keepdims=True) if kind == LAYER else v
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    return c * r, r


def normalise_grad(kind, vh, r, e):
    """Gradient with respect to v of sum(e * normalised(v))."""
    if kind == NONE:
        return e
    m = e.mean(-1, keepdims=True) if kind == LAYER else 0.0
    return r * (e - m - vh * (e * vh).mean(-1, keepdims=True))


def _per_sample(v, none):
    return none if v is None else v[:, None, :]


def residual_norm(h, y, post, pre, eps, alpha=1.0, gate=None, post_w=None, pre_w=None, scale=None, shift=None):
    """Rows [B, n, C] -> (h_out, x)."""
    out = alpha * h
    if y is not None:
        z = normalise(post, y, eps)[0] * (1.0 if post_w is None else post_w)
        out = out + _per_sample(gate, 1.0) * z
    x = normalise(pre, out, eps)[0] * (1.0 if pre_w is None else pre_w)
    return out, x * (1.0 + _per_sample(scale, 0.0)) + _per_sample(shift, 0.0)


def residual_norm_grad(h_out, y, dx, dh_out, post, pre, eps, alpha=1.0, gate=None, post_w=None, pre_w=None,
                       scale=None):
    """Gradients from the forward call's h_out and y: dict of dh, dy, dgate, dscale, dshift, dpost_w, dpre_w."""
    w, mod = (1.0 if pre_w is None else pre_w), 1.0 + _per_sample(scale, 0.0)
    dx = np.zeros_like(h_out) if dx is None else dx
    xh, r = normalise(pre, h_out, eps)
    dH = (0.0 if dh_out is None else dh_out) + normalise_grad(pre, xh, r, dx * w * mod)
    res = {"dh": alpha * dH, "dshift": dx.sum(1), "dscale": (dx * xh * w).sum(1), "dpre_w": (dx * xh * mod).sum((0, 1))}
    if y is not None:
        w, g = (1.0 if post_w is None else post_w), _per_sample(gate, 1.0)
        zh, rz = normalise(post, y, eps)
        res.update(dy=normalise_grad(post, zh, rz, dH * g * w), dgate=(dH * zh * w).sum(1),
                   dpost_w=(dH * zh * g).sum((0, 1)))
    return res


# ------------------------------------------------------------------ gated feed-forward
def activation(act, g):
    """(act(g), act'(g))."""
    if act == SILU:
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    k = np.sqrt(2.0 / np.pi)
    t = np.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)


def glu(x, w_gate, w_up, act):
    """Rows x [..., C], weights [F, C] -> (u, pre-activations g and w)."""
    g, w = x @ w_gate.T, x @ w_up.T
    return activation(act, g)[0] * w, g, w


def glu_grad(dy, x, w_gate, w_up, w_down, g, w, u, act):
    """Gradients of y = u w_down^T at the kept g, w and u; rows flattened ([R, ...])."""
    a, da = activation(act, g)
    du = dy @ w_down
    dg, dw = du * w * da, du * a
    return {"dx": dg @ w_gate + dw @ w_up, "dw_gate": dg.T @ x, "dw_up": dw.T @ x, "dw_down": dy.T @ u}
