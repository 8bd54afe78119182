"""The oracle's gradients of the gated block's layers against central differences
of its own forward functions, and its rotation against known angles (no GPU).

Central differences with step h = 1e-5 in float64 are good to about h^2 = 1e-10
of the third derivative plus 1e-16 / h = 1e-11 of the value; with values and
derivatives of order one, 1e-7 is safe."""
import numpy as np
import pytest

from oracle import layers


def _diff(f, v, h=1e-5):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        keep = v[i]
        v[i] = keep + h
        a = f()
        v[i] = keep - h
        b = f()
        v[i] = keep
        g[i] = (a - b) / (2 * h)
    return g


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
def test_residual_norm_grad_matches_differences(post, pre):
    rng = np.random.default_rng(10 * post + pre)
    B, n, C = 2, 3, 8
    v = {"h": rng.normal(size=(B, n, C)), "y": rng.normal(size=(B, n, C)), "gate": rng.normal(size=(B, C)),
         "scale": rng.normal(size=(B, C)), "shift": rng.normal(size=(B, C)), "post_w": rng.normal(size=C),
         "pre_w": rng.normal(size=C)}
    dh, dx = rng.normal(size=(B, n, C)), rng.normal(size=(B, n, C))

    def run():
        return layers.residual_norm(v["h"], v["y"], post, pre, 1e-3, 0.7, v["gate"], v["post_w"], v["pre_w"],
                                    v["scale"], v["shift"])

    def loss():
        h, x = run()
        return float((h * dh).sum() + (x * dx).sum())

    got = layers.residual_norm_grad(run()[0], v["y"], dx, dh, post, pre, 1e-3, 0.7, v["gate"], v["post_w"],
                                    v["pre_w"], v["scale"])
    for k in v:
        assert np.abs(got["d" + k] - _diff(loss, v[k])).max() < 1e-7, k


@pytest.mark.parametrize("act", [0, 1])
def test_glu_grad_matches_differences(act):
    rng = np.random.default_rng(act)
    x, dy = rng.normal(size=(4, 6)), rng.normal(size=(4, 3))
    w_gate, w_up, w_down = rng.normal(size=(5, 6)), rng.normal(size=(5, 6)), rng.normal(size=(3, 5))

    def loss():
        return float((layers.glu(x, w_gate, w_up, act)[0] @ w_down.T * dy).sum())

    u, g, w = layers.glu(x, w_gate, w_up, act)
    got = layers.glu_grad(dy, x, w_gate, w_up, w_down, g, w, u, act)
    for k, v in (("dx", x), ("dw_gate", w_gate), ("dw_up", w_up), ("dw_down", w_down)):
        assert np.abs(got[k] - _diff(loss, v)).max() < 1e-7, k


def test_rope_axes_turns_each_axis_by_its_own_coordinate():
    x = np.zeros((1, 1, 1, 10))
    x[..., 0::2] = 1.0
    pos = np.array([[0.5, -3.0]])
    y = layers.rope_axes(x, pos, (4, 4), base=100.0)[0, 0, 0]
    for i, ang in enumerate([0.5, 0.5 / 10, -3.0, -0.3]):
        assert np.allclose(y[2 * i:2 * i + 2], [np.cos(ang), np.sin(ang)], atol=1e-14)
    assert list(y[8:]) == [1.0, 0.0]
    rng = np.random.default_rng(0)
    x = rng.normal(size=(2, 3, 5, 10))
    pos = rng.normal(size=(2, 5, 2)) * 50
    back = layers.rope_axes(layers.rope_axes(x, pos, (4, 4)), pos, (4, 4), inverse=True)
    assert np.abs(back - x).max() < 1e-12
    # the inverse is the gradient: <dy, R x> = <R^-1 dy, x>
    dy = rng.normal(size=x.shape)
    assert abs((dy * layers.rope_axes(x, pos, (4, 4))).sum() - (layers.rope_axes(dy, pos, (4, 4), inverse=True) * x).sum()) < 1e-10
