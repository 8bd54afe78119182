"""The gated block's layers as torch.autograd functions.

Forward and backward run in librefadapt.so (refadapt_glu, refadapt_residual_norm,
refadapt_rope_axes and their backward passes); torch keeps the graph, allocates
the results and supplies the stream. bf16 rows and weights, fp32 vectors, on one
GPU; shapes as in ``api``. Gradients of bf16 tensors are bf16, of fp32 vectors
fp32. ``rope_axes`` can be differentiated any number of times (its gradient is the
inverse turn); the other two once: a second time raises."""
import functools

import torch

from . import api
from ._lib import RA_EPI_STORE

__all__ = ["gated_feed_forward", "residual_norm", "rope_axes"]


# Gradients come in whatever layout the graph gave them (transposed, strides of zero,
# part of a flat tensor at any offset); the calls want whole 16-byte pieces.
def _rows(grad):
    grad = grad.contiguous()
    return grad if grad.data_ptr() % 16 == 0 else grad.clone()


def _heads(grad):
    """[B, H, n, d]: any order of the axes but the last."""
    if grad.stride(3) == 1 and all(s % 8 == 0 for s in grad.stride()[:3]) and grad.data_ptr() % 16 == 0:
        return grad
    return grad.clone(memory_format=torch.contiguous_format)


class _Gradients(torch.autograd.Function):
    """The first n tensors, gradients that a kernel computed from the others."""

    @staticmethod
    def forward(ctx, n, *tensors):
        return tensors[:n]

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("gated_feed_forward and residual_norm cannot be differentiated twice")


def _once(backward):
    """A backward pass without a derivative of its own. Under create_graph its results stay
    connected to what they came from, so that a second derivative through them raises
    (torch's once_differentiable ties them to nothing: torch.autograd.grad then drops their
    part without a word)."""
    @functools.wraps(backward)
    def wrapper(ctx, *grads):
        with torch.no_grad():
            out = list(backward(ctx, *grads))
        if torch.is_grad_enabled():
            given = [i for i, v in enumerate(out) if v is not None]
            made = _Gradients.apply(len(given), *(out[i] for i in given),
                                    *(t for t in (*grads, *ctx.saved_tensors) if t is not None)) if given else ()
            for i, v in zip(given, made):
                out[i] = v
        return tuple(out)
    return wrapper


class _GatedFeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act, err_word, learn):
        B, n, C = x.shape
        F, O = w_gate.shape[0], w_down.shape[0]
        hidden, pre_gate, pre_up = (torch.empty((B, n, F), dtype=x.dtype, device=x.device) if need else None
                                    for need in (True, learn, learn))
        y = torch.empty((B, n, O), dtype=x.dtype, device=x.device)
        api.refadapt_glu([{"x": x, "w_gate": w_gate, "w_up": w_up, "out": hidden, "pre_gate": pre_gate,
                           "pre_up": pre_up}], F, C, act, err_word=err_word)
        api.refadapt_gemm([{"a": hidden, "w": w_down, "out": y}], O, F, RA_EPI_STORE, err_word=err_word)
        ctx.save_for_backward(x, w_gate, w_up, w_down, pre_gate, pre_up, hidden)
        ctx.act, ctx.err_word = act, err_word
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, pre_gate, pre_up, hidden = ctx.saved_tensors
        grads = [torch.empty_like(t, memory_format=torch.contiguous_format) if need else None
                 for t, need in zip((x, w_gate, w_up, w_down), ctx.needs_input_grad)]
        if any(g is not None for g in grads):
            ws = api.glu_backward_workspace(x.shape[0], x.shape[1], x.shape[2], w_gate.shape[0], w_down.shape[0],
                                            x.device)
            api.refadapt_glu_backward(_rows(dy), x, w_gate, w_up, w_down, pre_gate, pre_up, hidden, ctx.act, ws,
                                      dx=grads[0], dw_gate=grads[1], dw_up=grads[2], dw_down=grads[3],
                                      err_word=ctx.err_word)
        return (*grads, None, None, None)


def gated_feed_forward(x, w_gate, w_up, w_down, act, err_word=None):
    """(act(x w_gate^T) o (x w_up^T)) w_down^T: x [B, rows, C], w_gate and w_up
    [F, C], w_down [O, F], bf16 (F a multiple of 64, O of 256, which
    refadapt_gemm needs)."""
    # The pre-activations (twice the hidden rows) are kept for x, w_gate and w_up only.
    learn = torch.is_grad_enabled() and any(t.requires_grad for t in (x, w_gate, w_up))
    return _GatedFeedForward.apply(x, w_gate, w_up, w_down, act, err_word, learn)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, y, gate, post_w, pre_w, scale, shift, post, pre, eps, alpha, err_word):
        h_out, x = torch.empty_like(h), torch.empty_like(h)
        api.refadapt_residual_norm([{"h": h, "y": y, "h_out": h_out, "x": x, "gate": gate, "post_w": post_w,
                                     "pre_w": pre_w, "scale": scale, "shift": shift}], h.shape[2], post, pre, eps,
                                   alpha)
        ctx.save_for_backward(h_out, y, gate, post_w, pre_w, scale, shift)
        ctx.args = (post, pre, eps, alpha, err_word)
        return h_out, x

    @staticmethod
    @_once
    def backward(ctx, dh_out, dx):
        h_out, y, gate, post_w, pre_w, scale, shift = ctx.saved_tensors
        post, pre, eps, alpha, err_word = ctx.args
        B, n, C = h_out.shape
        seg = {"h": h_out, "y": y, "dx": _rows(dx), "dh_out": _rows(dh_out), "gate": gate,
               "post_w": post_w, "pre_w": pre_w, "scale": scale}
        grads = []
        for name, t, need in zip(("dh", "dy", "dgate", "dpost_w", "dpre_w", "dscale", "dshift"),
                                 (h_out, y, gate, post_w, pre_w, scale, shift), ctx.needs_input_grad):
            g = torch.empty_like(t, memory_format=torch.contiguous_format) if need and t is not None else None
            seg[name] = g
            grads.append(g)
        ws = api.residual_norm_backward_workspace(B, n, C, h_out.device)
        api.refadapt_residual_norm_backward(seg, C, post, pre, ws, eps, alpha, err_word)
        return (*grads, None, None, None, None, None)


def residual_norm(h, y, post, pre, gate=None, post_w=None, pre_w=None, scale=None, shift=None, eps=1e-6, alpha=1.0,
                  err_word=None):
    """(h_out, x): h_out = alpha h + gate N_post(y) post_w, x = N_pre(h_out)
    pre_w (1 + scale) + shift. h, y [B, rows, C] bf16 (y may be None); gate,
    scale, shift [B, C], post_w, pre_w [C] fp32 or None. Without y, gate and
    post_w have no part in the result."""
    if y is None:
        gate = post_w = None
    return _ResidualNorm.apply(h, y, gate, post_w, pre_w, scale, shift, post, pre, eps, alpha, err_word)


class _RopeAxes(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, axes, base, inverse):
        out = torch.empty_like(x)
        api.refadapt_rope_axes([(x, out)], pos, axes, base, inverse=inverse)
        ctx.save_for_backward(pos)
        ctx.args = (axes, base, inverse)
        return out

    @staticmethod
    def backward(ctx, dout):
        (pos,) = ctx.saved_tensors
        axes, base, inverse = ctx.args
        return _RopeAxes.apply(_heads(dout), pos, axes, base, not inverse), None, None, None, None


def rope_axes(x, pos, axes, base=10000.0):
    """x [B, H, n, d] bf16 turned by the rows' coordinates pos ([n, len(axes)] or [B, n, len(axes)] fp32)."""
    return _RopeAxes.apply(x, pos, tuple(axes), base, False)
