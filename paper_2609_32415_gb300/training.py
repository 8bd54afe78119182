"""The gated block's layers as torch.autograd functions, linear layers through 4-bit
products, and the optimiser.

Forward and backward run in librefadapt.so (refadapt_glu, refadapt_residual_norm,
refadapt_rope_axes, refadapt_quant4 with refadapt_gemm4, and their backward passes);
torch keeps the graph, allocates the results and supplies the stream. bf16 rows and
weights, fp32 vectors, on one GPU; shapes as in ``api``. Gradients of bf16 tensors are
bf16, of fp32 vectors fp32. ``rope_axes`` can be differentiated any number of times (its
gradient is the inverse turn); the others once: a second time raises. ``AdamW`` steps
over all parameters in one call (refadapt_grad_norm, refadapt_adamw)."""
import functools
import math

import torch

from . import api
from ._lib import RA_EPI_STORE, RA_Q4_E8M0

__all__ = ["gated_feed_forward", "residual_norm", "rope_axes", "linear4", "AdamW"]


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
        raise RuntimeError("gated_feed_forward, residual_norm and linear4 cannot be differentiated twice")


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


class _Linear4(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, format, x_exponent, w_exponent, err_word):
        (B, n, K), N = x.shape, w.shape[0]
        y = torch.empty((B, n, N), dtype=x.dtype, device=x.device)
        w4 = api.weight4(w, format, w_exponent)
        codes, scales = api.quant4_buffers(B, n, K, format, x.device)
        api.refadapt_quant4([{"x": x, "codes": codes, "scales": scales, "exponent": x_exponent}], K, format)
        api.refadapt_gemm4([{"a": codes, "a_scales": scales, "a_exponent": x_exponent, "w": w4.codes,
                             "w_scales": w4.scales, "w_exponent": w4.exponent, "out": y}], N, K, RA_EPI_STORE, format,
                           err_word=err_word)
        ctx.save_for_backward(x, w)
        ctx.err_word = err_word
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        dx, dw = (torch.empty_like(t, memory_format=torch.contiguous_format) if need else None
                  for t, need in zip((x, w), ctx.needs_input_grad))
        if dx is not None or dw is not None:
            ws = api.linear4_backward_workspace(x.shape[0], x.shape[1], x.shape[2], w.shape[0], x.device)
            # the product takes weights in rows of any stride, their gradient whole ones
            api.refadapt_linear4_backward(_rows(dy), x, w.contiguous(), ws, dx=dx, dw=dw, err_word=ctx.err_word)
        return dx, dw, None, None, None, None


def linear4(x, w, format=RA_Q4_E8M0, x_exponent=0, w_exponent=0, err_word=None):
    """x w^T through 4-bit products, x [B, rows, K], w [N, K] bf16 (N and K multiples of
    64; rows of a wider buffer are fine): forward in the format given, the gradients in RA_Q4_E8M0,
    which has no range to choose. RA_Q4_E4M3 has one for x and one for w: scales (a block's
    largest magnitude / 6) are within 1 / 16 from 2^(exponent - 6) to 448 2^exponent, so that
    w_exponent 0 suits blocks that reach 0.1 to 2688; None takes api.weight4's, from the weight's
    largest magnitude (which waits for the GPU). Rounding to 4 bits counts as the identity
    in the backward pass."""
    return _Linear4.apply(x, w, format, x_exponent, w_exponent, err_word)


class AdamW:
    """AdamW over a list of parameters (contiguous, fp32 or bf16; bf16 ones get an fp32
    copy, made here, that the steps add up in: load weights first), with clipping to max_norm. bits: 32 or 8, of the
    moments. capturable: the rate lives on the GPU too (``lr``, fp32), so that a captured
    step goes on when it is replayed. A step whose gradients' norm (refadapt_grad_norm's) is
    not finite changes no parameter and does not count. ``count`` is the number of the steps that did:
    an int32 tensor with capturable, else an int (reading it waits for the GPU). ``norm`` holds the last
    step's gradient norm and clipping factor (on the GPU)."""

    def __init__(self, params, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32, max_norm=math.inf, seed=0,
                 capturable=False):
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamW: no parameters")
        if len({id(p) for p in self.params}) < len(self.params):
            raise ValueError("AdamW: a parameter twice")
        for p in self.params:
            if p.dtype not in (torch.float32, torch.bfloat16) or not p.is_cuda or not p.is_contiguous():
                raise ValueError("AdamW: expected contiguous fp32 or bf16 CUDA parameters, got %s %s %s"
                                 % (tuple(p.shape), p.dtype, p.device))
        dev = self.params[0].device
        self.betas, self.eps, self.weight_decay, self.max_norm, self.seed = betas, eps, weight_decay, max_norm, seed
        self.bits, self.capturable = bits, capturable
        self.lr = torch.tensor([lr], dtype=torch.float32, device=dev) if capturable else lr
        self.state = [dict(api.adamw_moments(p, bits), **({} if p.dtype == torch.float32 else {"p": p.detach().float()}))
                      for p in self.params]
        self.norm = torch.zeros(2, dtype=torch.float32, device=dev)
        self._factor = self.norm[1:]
        self._workspace = api.grad_norm_workspace(dev)
        self._count = self._workspace[4:8].view(torch.int32)  # norms that were finite

    @property
    def count(self):
        return self._count if self.capturable else int(self._count)

    @count.setter
    def count(self, value):
        self._count.copy_(torch.as_tensor(value, dtype=torch.int32).reshape(1))

    def zero_grad(self, set_to_none=True):
        for p in self.params:
            if set_to_none:
                p.grad = None
            elif p.grad is not None:
                p.grad.detach_().zero_()

    @torch.no_grad()
    def step(self):
        tensors = []
        for p, state in zip(self.params, self.state):
            if p.grad is None:
                continue
            g = p.grad.contiguous()
            tensors.append({"p": p, "g": g, **state} if p.dtype == torch.float32 else {"g": g, "w": p, **state})
        api.refadapt_grad_norm([t["g"] for t in tensors], self.max_norm, self.norm, self._workspace)
        try:
            api.refadapt_adamw(tensors, self.lr, self._count, beta1=self.betas[0], beta2=self.betas[1], eps=self.eps,
                               weight_decay=self.weight_decay, grad_scale=self._factor, seed=self.seed)
        except Exception:  # refused: nothing has changed (the factor of a norm that is not finite is NaN)
            self._count.sub_((self._factor >= 0).int())
            raise
        # written behind torch's back: a graph that saved one of them must not use it any more
        torch.autograd.graph.increment_version([t["w"] if "w" in t else t["p"] for t in tensors])

    def state_dict(self):
        """The moments, the fp32 copies and the step's number (the tensors themselves)."""
        return {"state": self.state, "count": self.count, "bits": self.bits}

    def load_state_dict(self, saved):
        if saved["bits"] != self.bits or len(saved["state"]) != len(self.state):
            raise ValueError("AdamW: a state of %d tensors in %d bits for %d in %d"
                             % (len(saved["state"]), saved["bits"], len(self.state), self.bits))
        for mine, theirs in zip(self.state, saved["state"]):
            if {k: (v.shape, v.dtype) for k, v in mine.items()} != {k: (v.shape, v.dtype) for k, v in theirs.items()}:
                raise ValueError("AdamW: a state of other shapes or types")
        for mine, theirs in zip(self.state, saved["state"]):
            for k, v in mine.items():
                v.view(torch.uint8).copy_(theirs[k].view(torch.uint8)) if v.element_size() == 1 else v.copy_(theirs[k])
        self.count = saved["count"]
