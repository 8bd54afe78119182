"""The autograd functions of the gated block's layers inside torch's graph: gradients
that arrive in every layout torch hands on, second derivatives, calls that keep
nothing for a backward pass, and inputs that a call does not use.

Tolerances are those of test_gpu_block_layers (one rounding to bf16) where an
operator's backward call is compared on the gradient that it was given; a graph's own
gradients carry bf16 tensors between layers: a few 2^-9 normwise, 1e-2 has room."""
import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import layers
from test_gpu_block_layers import bf, close, d64, f32

pytestmark = pytest.mark.gpu


def relative(a, b):
    return float((a.double() - b).norm() / (b.norm() + 1e-300))


# ------------------------------------------------------------------ layouts of gradients
def rope_loss(layout, y, g):
    """A loss whose gradient with respect to y ([B, H, n, d]) arrives in the layout."""
    B, H, n, d = y.shape
    if layout == "product":      # that of k in q @ k^T: the last axis is not contiguous
        return (bf((B, H, n, d), g) @ y.transpose(-1, -2)).float().square().sum()
    if layout == "sum":          # one number for all elements: strides of zero
        return y.sum()
    if layout == "sum of rows":  # strides of zero but for the last axis
        return (y.sum((0, 1, 2)).float() * f32((d,), g)).sum()
    if layout == "odd offset":   # part of a flat tensor, three elements in: not 16-byte aligned
        z = torch.cat((y.new_zeros(3), y.reshape(-1)))
        return (z * bf(z.shape, g)).float().sum()
    assert layout == "token"     # token-major, taken as it is
    z = y.transpose(1, 2)
    return (z * bf(z.shape, g)).float().sum()


@pytest.mark.parametrize("layout", ["product", "sum", "sum of rows", "odd offset", "token"])
def test_rope_gradient_in_every_layout(cuda_ok, layout):
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(len(layout))
    B, H, n, d, axes = 2, 4, 75, 64, (24, 32)
    x = bf((B, H, n, d), g).requires_grad_(True)
    pos = f32((n, 2), g, 20.0)
    y = training.rope_axes(x, pos, axes)
    given = []
    y.register_hook(lambda v: given.append(v.clone()))
    rope_loss(layout, y, g).backward()
    ref = layers.rope_axes(f64(given[0]), d64(pos), axes, inverse=True)
    ok, worst = close(f64(x.grad), ref, np.abs(f64(given[0])).max())
    assert ok, worst


def test_row_gradients_that_are_not_aligned(cuda_ok):
    """The other two functions, with gradients that start three elements into a flat tensor."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(7)
    B, n, C, F = 2, 33, 256, 128
    leaves = [bf((B, n, C), g).requires_grad_(True), bf((B, n, C), g).requires_grad_(True)]
    w = [bf((F, C), g, C ** -0.5), bf((F, C), g, C ** -0.5), bf((C, F), g, F ** -0.5)]
    up = [bf((3 + B * n * C,), g) for _ in range(3)]

    def grads(shift):
        h, x = training.residual_norm(leaves[0], leaves[1], 2, 1)
        y = training.gated_feed_forward(leaves[0], *w, 0)
        loss = 0.0
        for t, u in zip((h, x, y), up):
            t = torch.cat((t.new_zeros(3), t.reshape(-1))) if shift else t.reshape(-1)
            loss = loss + (t * (u if shift else u[3:].clone())).float().sum()
        return torch.autograd.grad(loss, leaves)

    for a, b in zip(grads(True), grads(False)):
        assert torch.equal(a, b)


# ------------------------------------------------------------------ second derivatives
def test_rope_is_differentiable_twice(cuda_ok):
    """d/dx of |d(sum rope(x)^2 u)/dx|^2: the gradient passes through the backward call."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(11)
    B, H, n, d, axes = 1, 2, 40, 64, (32, 32)
    x, u, pos = bf((B, H, n, d), g).requires_grad_(True), f32((B, H, n, d), g), f32((n, 2), g, 5.0)
    y = training.rope_axes(x, pos, axes)
    (first,) = torch.autograd.grad((y.float() ** 2 * u).sum(), x, create_graph=True)
    (got,) = torch.autograd.grad((first.float() ** 2).sum(), x)

    ang = torch.as_tensor(layers.rope_axes_angles(d64(pos), axes)).cuda()
    c, s = torch.cos(ang), torch.sin(ang)

    def turn(v):
        e, o = v[..., 0::2], v[..., 1::2]
        return torch.stack((e * c - o * s, e * s + o * c), -1).flatten(-2)

    x2 = x.detach().double().requires_grad_(True)
    (first2,) = torch.autograd.grad((turn(x2) ** 2 * u.double()).sum(), x2, create_graph=True)
    (want,) = torch.autograd.grad((first2 ** 2).sum(), x2)
    assert float(want.norm()) > 0 and relative(got, want) < 1e-2, relative(got, want)


@pytest.mark.parametrize("layer", ["feed-forward", "norm"])
def test_second_derivatives_are_refused_where_there_are_none(cuda_ok, layer):
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(12)
    x = bf((1, 20, 256), g).requires_grad_(True)
    if layer == "norm":
        _, y = training.residual_norm(x, None, 0, 2)
    else:
        y = training.gated_feed_forward(x, bf((64, 256), g, 0.06), bf((64, 256), g, 0.06), bf((256, 64), g, 0.1), 0)
    # 0.5 |y|^2 keeps a path to x besides the layer's backward call, so that the graph does not end at once
    (first,) = torch.autograd.grad(0.5 * (y.float() ** 2).sum() + (x.float() ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        torch.autograd.grad((first.float() ** 2).sum(), x)


# ------------------------------------------------------------------ what a call does not need
def test_feed_forward_keeps_nothing_where_nothing_is_learned(cuda_ok):
    """Without gradients a call has its result and the hidden rows only; with the down
    projection alone to learn it keeps no pre-activations either. The results are those of the
    call that keeps everything."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(13)
    n, C, F = 2048, 256, 4096
    x = bf((1, n, C), g)
    w = [bf((F, C), g, C ** -0.5), bf((F, C), g, C ** -0.5), bf((C, F), g, F ** -0.5)]

    def peak(f):
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        y = f()
        torch.cuda.synchronize()
        return y, torch.cuda.max_memory_allocated() - before

    hidden, small = 2 * n * F, 2 * n * C + (1 << 20)

    def call():
        return training.gated_feed_forward(x, *w, 0)

    frozen, bytes_frozen = peak(call)
    w[2].requires_grad_(True)
    down, bytes_down = peak(call)
    for t in (x, *w):
        t.requires_grad_(True)
    everything, bytes_all = peak(call)
    with torch.no_grad():
        without, bytes_without = peak(call)
    assert bytes_all >= 3 * hidden
    assert max(bytes_frozen, bytes_down, bytes_without) <= hidden + small, (bytes_frozen, bytes_down, bytes_without)
    for y in (frozen, down, without):
        assert torch.equal(y, everything)
    dy = bf(y.shape, g)
    (got,) = torch.autograd.grad(down, w[2], dy)
    (want,) = torch.autograd.grad(everything, w[2], dy)
    assert torch.equal(got, want)


def test_norm_without_a_branch_ignores_its_gate_and_weight(cuda_ok):
    """h_out = alpha h where y is absent: gate and post_w have no part in it, and no gradient."""
    from paper_2609_32415_gb300 import training
    g = torch.Generator().manual_seed(14)
    h = bf((2, 9, 64), g).requires_grad_(True)
    gate, post_w = f32((2, 64), g).requires_grad_(True), f32((64,), g).requires_grad_(True)
    pre_w = f32((64,), g, 0.1, 1.0).requires_grad_(True)
    up = f32((2, 9, 64), g)
    h_out, x = training.residual_norm(h, None, 2, 2, gate=gate, post_w=post_w, pre_w=pre_w)
    got = torch.autograd.grad((x.float() * up).sum() + h_out.float().sum(), (h, pre_w, gate, post_w), allow_unused=True)
    h_out, x = training.residual_norm(h, None, 2, 2, pre_w=pre_w)
    want = torch.autograd.grad((x.float() * up).sum() + h_out.float().sum(), (h, pre_w))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(v is None or not v.any() for v in got[2:])
