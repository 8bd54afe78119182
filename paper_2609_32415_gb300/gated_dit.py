"""Algorithm 1 over a stack of gated DiT blocks.

The same method and caches as ``DiTExecutor`` (see ``dit``) over blocks whose
layers around the joint attention are

  * rotary positions with several axes (time, height, width, ...) on q and k;
  * a norm before and a norm after each branch (LayerNorm or RMS norm, with or
    without weights), the branch's AdaLN gate between the latter and the
    residual sum;
  * a gated feed-forward act(x Wg^T) o (x Wu^T) with a down projection.

Per block and stream: x = N_pre(h) w_pre (1 + scale) + shift; attention or
feed-forward of x gives y; h <- h + gate N_post(y) w_post. The norm after a
branch, the gate, the residual sum and the norm before the next branch are one
call within a block. With resident weights (see ``step``) they are across the
border of two blocks too: a block's last call then also gives the next block's x
for the text and target rows (not for the reference rows, which wait for that
block's decision).
"""
import torch

from . import api
from ._lib import RA_ACT_GELU, RA_ACT_SILU, RA_EPI_STORE, RA_NORM_LAYER, RA_NORM_NONE, RA_NORM_RMS
from .dit import ROLES, STREAM_OF, DiTExecutor

NORMS = {"none": RA_NORM_NONE, "layer": RA_NORM_LAYER, "rms": RA_NORM_RMS}
ACTS = {"silu": RA_ACT_SILU, "gelu": RA_ACT_GELU}


class GatedDiTExecutor(DiTExecutor):
    """pos: [n_text + n_ref + n_tgt, len(axes)] fp32 coordinates of the joint
    rows; axes: columns of a head per axis; ff_width: features of the gated
    feed-forward (a multiple of 64); pre, post: "layer", "rms" or (post)
    "none". Weights per stream: w_qkv, b_qkv, q_norm, k_norm, w_o, b_o as for
    DiTExecutor; w_gate, w_up [F, C], w_2 [C, F] bf16, b_2 [C] fp32; optional
    norm weights pre_a, post_a, pre_m, post_m [C] fp32 (attention and
    feed-forward branch). With weights4 (see DiTExecutor) w_qkv, w_o and w_2 are
    api.Weight4; w_gate and w_up stay bf16."""

    def __init__(self, n_blocks, B, H, d, n_text, n_ref, n_tgt, theta, delta_max, pos, axes, ff_width, pre="rms",
                 post="rms", act="silu", rope_base=10000.0, device="cuda", **kw):
        for name, table, value in (("pre", NORMS, pre), ("post", NORMS, post), ("act", ACTS, act)):
            if value not in table:
                raise ValueError("unknown %s %r" % (name, value))
        if tuple(pos.shape) != (n_text + n_ref + n_tgt, len(axes)):
            raise ValueError("pos: expected [%d, %d] coordinates, got %s"
                             % (n_text + n_ref + n_tgt, len(axes), tuple(pos.shape)))
        super().__init__(n_blocks, B, H, d, n_text, n_ref, n_tgt, theta, delta_max, device=device, mlp_width=ff_width,
                         **kw)
        self.pre, self.post, self.act = NORMS[pre], NORMS[post], ACTS[act]
        dev = torch.device(device)
        self.rope = api.rope_axes_table(pos.to(device=dev, dtype=torch.float32).contiguous(), d, axes, rope_base)
        self.y = {r: torch.empty((B, self.n[r], self.C), dtype=torch.bfloat16, device=dev) for r in ROLES}
        self._next = None       # (mods, weights) of the block after this one, inside step()
        self._x_ready = False   # x of the text and target rows came with the last block

    def _norm(self, segs, mode, stream):
        api.refadapt_residual_norm(segs, self.C, self.post, self.pre, self.ln_eps, mode=mode, stream=stream)

    def _branch_input(self, roles, hin, ms, Ws, mode, stream):
        if self._x_ready and "ref" not in roles:
            return
        self._norm([{"h": hin[r], "x": self.x[r], "shift": ms[r]["shift_a"], "scale": ms[r]["scale_a"],
                     "pre_w": Ws[r].get("pre_a"), "gated": r == "ref"} for r in roles], mode, stream)

    def _finish_block(self, t, b, hin, ms, Ws, mode, stream):
        C, F = self.C, self.F
        self._gemm("o_proj", t, b, [
            {"a": self.o[r], "w": Ws[r]["w_o"], "bias": Ws[r]["b_o"], "out": self.y[r], "gated": r == "ref"}
            for r in ROLES], C, C, RA_EPI_STORE, mode=mode, err_word=self.err, stream=stream)
        self._norm([{"h": hin[r], "y": self.y[r], "gate": ms[r]["gate_a"], "post_w": Ws[r].get("post_a"),
                     "h_out": self.h1[r], "x": self.x[r], "shift": ms[r]["shift_m"], "scale": ms[r]["scale_m"],
                     "pre_w": Ws[r].get("pre_m"), "gated": r == "ref"} for r in ROLES], mode, stream)
        api.refadapt_glu([{"x": self.x[r], "w_gate": Ws[r]["w_gate"], "w_up": Ws[r]["w_up"], "out": self.u[r],
                           "gated": r == "ref"} for r in ROLES], F, C, self.act, mode=mode, err_word=self.err,
                         stream=stream)
        self._gemm("ff_down", t, b, [
            {"a": self.u[r], "w": Ws[r]["w_2"], "bias": Ws[r]["b_2"], "out": self.y[r], "gated": r == "ref"}
            for r in ROLES], C, F, RA_EPI_STORE, mode=mode, err_word=self.err, stream=stream)
        out = {"text": self.h["text"], "ref": self.hbar[b + 1], "tgt": self.h["tgt"]}
        segs = []
        for r in ROLES:
            s = {"h": self.h1[r], "y": self.y[r], "gate": ms[r]["gate_m"], "post_w": Ws[r].get("post_m"),
                 "h_out": out[r], "gated": r == "ref"}
            if self._next is not None and r != "ref":
                m, w = (v[STREAM_OF[r]] for v in self._next)
                s.update(x=self.x[r], shift=m["shift_a"], scale=m["scale_a"], pre_w=w.get("pre_a"))
            segs.append(s)
        self._norm(segs, mode, stream)

    def step(self, t, h_in, mods, weights, log_index=None, stream=None, after_block=None, resident=False):
        """As DiTExecutor.step. resident: what mods and weights give stays valid, unchanged,
        until the step's work has run, and they may be asked for a block before the one in
        front of it is enqueued; the border of two blocks is then one call (x of the next
        block from the unrounded rows), unless an after_block hook stands on it."""
        if not resident or after_block is not None:
            return super().step(t, h_in, mods, weights, log_index, stream, after_block)
        self.hbar[0] = h_in["ref"]
        here = (mods(t, 0), weights(0))
        try:
            for b in range(self.n_blocks):
                src = {"text": h_in["text"], "tgt": h_in["tgt"]} if b == 0 else self.h
                self._next = (mods(t, b + 1), weights(b + 1)) if b + 1 < self.n_blocks else None
                self._x_ready = b > 0
                self.block(t, b, src, here[0], here[1], log_index, stream)
                here = self._next
        finally:
            self._next, self._x_ready = None, False
