"""Thin Python binding of the C ABI (include/refadapt.h), same names.

Only argument marshalling happens here (natively, csrc/binding.cpp, for the
calls of a step): torch tensors supply device memory and streams; every step
of the computation runs in librefadapt.so's kernels.
Tensors are [B, H, n, d] bf16 CUDA views with a contiguous last axis (any
other strides, 16-byte aligned).
"""
import collections
import ctypes
import math

import torch

from . import _lib
from ._lib import RA_Q4_E4M3, RA_Q4_E8M0, RaSeg, check

__all__ = ["seg", "refadapt_joint_attn", "refadapt_mass_partial_len", "refadapt_q_delta",
           "refadapt_q_delta_workspace_size", "refadapt_q_delta_noalloc", "refadapt_state_size", "refadapt_state_init",
           "refadapt_gate", "refadapt_ref_cache_update", "refadapt_set_wait_budget_ns",
           "refadapt_check_error", "refadapt_version", "refadapt_last_launch", "refadapt_selftest_wait_timeout", "q_delta_workspace", "new_state",
           "alloc_mass_partial", "refadapt_rope_table", "rope_table", "refadapt_ln_modulate", "refadapt_gemm",
           "refadapt_rope_axes", "refadapt_rope_axes_table", "rope_axes_table", "refadapt_residual_norm",
           "refadapt_residual_norm_backward", "refadapt_residual_norm_backward_workspace_size",
           "residual_norm_backward_workspace", "refadapt_glu", "refadapt_glu_backward",
           "refadapt_glu_backward_workspace_size", "glu_backward_workspace", "Weight4", "weight4", "quant4_buffers",
           "refadapt_quant4", "refadapt_quant4_scales_size", "refadapt_gemm4", "refadapt_linear4_backward",
           "refadapt_linear4_backward_workspace_size", "linear4_backward_workspace", "refadapt_grad_norm",
           "refadapt_grad_norm_workspace_size", "grad_norm_workspace", "refadapt_adamw", "adamw_moments"]


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _handle(stream):
    """A stream argument for the native calls: None (the current stream) or the raw handle."""
    if stream is None:
        return None
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def seg(t, n=None) -> RaSeg:
    """ra_seg of a [B, H, n, d] bf16 CUDA tensor (None -> empty/absent segment)."""
    if t is None:
        return RaSeg(None, 0, 0, 0, int(n or 0), 0)
    if t.dim() != 4 or t.dtype != torch.bfloat16 or not t.is_cuda or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("expected a [B, H, n, d] bf16 CUDA tensor with contiguous last axis, got %s %s %s"
                         % (tuple(t.shape), t.dtype, t.device))
    ptr = t.data_ptr() if t.numel() > 0 else 0
    return RaSeg(ptr or None, t.stride(0), t.stride(1), t.stride(2), t.shape[2], 0)


def refadapt_mass_partial_len(n_text, n_tgt) -> int:
    return int(_lib.load().refadapt_mass_partial_len(int(n_text), int(n_tgt)))


def alloc_mass_partial(B, H, n_text, n_tgt, device="cuda"):
    return torch.zeros((B, H, refadapt_mass_partial_len(n_text, n_tgt)), dtype=torch.float32, device=device)


def refadapt_joint_attn(q, k, v, o, mass_partial, mode=None, softmax_scale=0.0, ref_logit_bias=None,
                        mass_rows=0, err_word=None, mass_row_stride=0, ref_fresh=None, a_b=None, step=0,
                        stream=None):
    """q, k, v, o: sequences (text, ref, tgt) of [B, H, n, d] tensors; q[1] / o[1] may be None.
    ref_fresh: optional (q, k, v) of this step's reference rows for the fused
    cache update (q may be None when q[1] is); a_b, step: the stamp it writes."""
    if ref_fresh is None and a_b is not None:
        raise ValueError("refadapt_joint_attn: a_b is written only with ref_fresh")
    return check("refadapt_joint_attn", _lib.native().joint_attn(
        q, k, v, o, mass_partial, mode, float(softmax_scale), ref_logit_bias, int(mass_rows), err_word,
        int(mass_row_stride), ref_fresh, a_b, int(step), _handle(stream)))


def refadapt_q_delta_workspace_size(B, H) -> int:
    return int(_lib.load().refadapt_q_delta_workspace_size(int(B), int(H)))


def q_delta_workspace(B, H, device="cuda"):
    """A zero-filled workspace for refadapt_q_delta (reusable across calls)."""
    return torch.zeros(refadapt_q_delta_workspace_size(B, H), dtype=torch.uint8, device=device)


def refadapt_q_delta(q_cur, q_prev, d_out, workspace, eps=1e-6, stream=None):
    return check("refadapt_q_delta", _lib.native().q_delta(q_cur, q_prev, d_out, workspace, float(eps),
                                                           _handle(stream)))


def refadapt_q_delta_noalloc(q_cur, q_prev, d_out, eps=1e-6, stream=None):
    """refadapt_q_delta without a workspace (static scratch inside the library;
    B * H <= RA_Q_DELTA_NOALLOC_MAX_BH; calls must not overlap on the GPU)."""
    lib = _lib.load()
    B, H, _, d = q_cur.shape
    sc, sp = seg(q_cur), seg(q_prev)
    return check("refadapt_q_delta_noalloc", lib.refadapt_q_delta_noalloc(
        ctypes.byref(sc), ctypes.byref(sp), B, H, d, float(eps), _ptr(d_out), _stream(stream)))


def refadapt_state_size(B) -> int:
    return int(_lib.load().refadapt_state_size(int(B)))


def refadapt_state_init(state, B, stream=None):
    return check("refadapt_state_init", _lib.load().refadapt_state_init(_ptr(state), int(B), _stream(stream)))


def new_state(B, device="cuda", stream=None):
    st = torch.empty(refadapt_state_size(B), dtype=torch.uint8, device=device)
    refadapt_state_init(st, B, stream)
    return st


def refadapt_gate(t, b, state, mode_out, theta, delta_max, B, H, q_delta=None, mass_partial_prev=None,
                  mass_row_count=0, forced_boundary=-1, gbar_out=None, m_out=None, cue=0, stream=None):
    return check("refadapt_gate", _lib.native().gate(
        int(t), int(b), state, mode_out, float(theta), int(delta_max), int(B), int(H), q_delta, mass_partial_prev,
        int(mass_row_count), int(forced_boundary), gbar_out, m_out, int(cue), _handle(stream)))


def refadapt_q_delta_gate(q_cur, q_prev, d_out, workspace, t, b, state, mode_out, theta, delta_max,
                          mass_partial_prev, mass_row_count, eps=1e-6, forced_boundary=-1, gbar_out=None,
                          m_out=None, cue=0, stream=None):
    """refadapt_q_delta then refadapt_gate on its D (t >= 1), in one launch
    when the Q change takes its cluster path."""
    return check("refadapt_q_delta_gate", _lib.native().q_delta_gate(
        q_cur, q_prev, d_out, workspace, float(eps), _handle(stream), int(t), int(b), state, mode_out, float(theta),
        int(delta_max), mass_partial_prev, int(mass_row_count), int(forced_boundary), gbar_out, m_out, int(cue)))


def refadapt_ref_cache_update(k_src, v_src, k_cache, v_cache, mode, t, a_b=None, x_src=None, x_cache=None,
                              stream=None):
    lib = _lib.load()
    B, H, _, d = k_src.shape
    ks, vs, kc, vc = seg(k_src), seg(v_src), seg(k_cache), seg(v_cache)
    if x_src is not None:
        xs, xc = seg(x_src), seg(x_cache)
        xp, xcp = ctypes.byref(xs), ctypes.byref(xc)
        x_heads, x_width = x_src.shape[1], x_src.shape[3]
    else:
        xp = xcp = None
        x_heads = x_width = 0
    return check("refadapt_ref_cache_update", lib.refadapt_ref_cache_update(
        ctypes.byref(ks), ctypes.byref(vs), ctypes.byref(kc), ctypes.byref(vc), B, H, d, xp, xcp,
        x_heads, x_width, _ptr(mode), int(t), _ptr(a_b), _stream(stream)))


def refadapt_set_wait_budget_ns(ns):
    _lib.load().refadapt_set_wait_budget_ns(int(ns))


def refadapt_check_error(err_word, stream=None):
    return check("refadapt_check_error", _lib.load().refadapt_check_error(_ptr(err_word), _stream(stream)))


def refadapt_selftest_wait_timeout(err_word, budget_ns, stream=None):
    return check("refadapt_selftest_wait_timeout",
                 _lib.load().refadapt_selftest_wait_timeout(_ptr(err_word), int(budget_ns), _stream(stream)))


def refadapt_last_launch() -> str:
    return _lib.load().refadapt_last_launch().decode()


def refadapt_version() -> int:
    return int(_lib.load().refadapt_version())


# --------------------------------------------------------------------------- DiT block around the attention
def refadapt_rope_table(table, n_pos, d, base=10000.0, stream=None):
    return check("refadapt_rope_table", _lib.load().refadapt_rope_table(
        _ptr(table), int(n_pos), int(d), float(base), _stream(stream)))


def rope_table(n_pos, d, base=10000.0, device="cuda", stream=None):
    """[n_pos, d/2, 2] fp32 (cos, sin) table built by refadapt_rope_table."""
    t = torch.empty((int(n_pos), int(d) // 2, 2), dtype=torch.float32, device=device)
    refadapt_rope_table(t, n_pos, d, base, stream)
    return t


def refadapt_ln_modulate(segs, C, eps=1e-6, mode=None, stream=None):
    """segs: up to three dicts with h, x ([B, rows, C] bf16), shift, scale
    ([B, C] fp32) and optional gated (bool)."""
    return check("refadapt_ln_modulate",
                 _lib.native().ln_modulate(segs, int(C), float(eps), mode, _handle(stream)))


def refadapt_gemm(segs, N, K, epilogue, mode=None, rope=None, H=0, d=0, norm_eps=1e-6, err_word=None,
                  tile_mode=0, stream=None):
    """segs: up to three dicts with a ([B, rows, K] bf16), w ([N, K] bf16),
    optional bias ([N] fp32), gated; plus per epilogue out ([B, rows, N]),
    resid and gate ([B, N] fp32) for RESID, or q, k, v ([B, H, rows, d]),
    q_norm, k_norm ([d] fp32) and pos_offset for QKV."""
    return check("refadapt_gemm", _lib.native().gemm(
        segs, int(N), int(K), int(epilogue), mode, rope, int(H), int(d), float(norm_eps), err_word, int(tile_mode),
        _handle(stream)))


# --------------------------------------------------------------------------- layers of gated DiT blocks
def refadapt_rope_axes(tensors, pos, axes, base=10000.0, inverse=False, stream=None):
    """Rotary positions with several axes. tensors: one or two (x, out) pairs of
    [B, H, n, d] bf16 (out may be x); pos: [n, len(axes)] or [B, n, len(axes)]
    fp32 coordinates; axes: columns of a head per axis. inverse: the backward
    pass (turns by the negative angle)."""
    return check("refadapt_rope_axes", _lib.native().rope_axes(tensors, pos, axes, float(base), bool(inverse),
                                                               _handle(stream)))


def refadapt_rope_axes_table(table, pos, axes, base=10000.0, stream=None):
    """Fills table ([n, d/2, 2] fp32) for refadapt_gemm's QKV epilogue from pos ([n, len(axes)] fp32)."""
    n, pairs = _axes_table_shape(table, pos, axes)
    dims = (ctypes.c_int32 * len(axes))(*[int(a) for a in axes])
    return check("refadapt_rope_axes_table", _lib.load().refadapt_rope_axes_table(
        _ptr(table), _ptr(pos), n, 2 * pairs, len(axes), dims, float(base), _stream(stream)))


def _axes_table_shape(table, pos, axes):
    if pos.dim() != 2 or pos.dtype != torch.float32 or not pos.is_cuda or not pos.is_contiguous() or \
            pos.shape[1] != len(axes):
        raise ValueError("pos: expected a contiguous [n, %d] fp32 CUDA tensor, got %s %s %s"
                         % (len(axes), tuple(pos.shape), pos.dtype, pos.device))
    if table.dim() != 3 or table.dtype != torch.float32 or not table.is_cuda or not table.is_contiguous() or \
            table.shape[0] != pos.shape[0] or table.shape[2] != 2:
        raise ValueError("table: expected a contiguous [%d, d/2, 2] fp32 CUDA tensor, got %s %s %s"
                         % (pos.shape[0], tuple(table.shape), table.dtype, table.device))
    return table.shape[0], table.shape[1]


def rope_axes_table(pos, d, axes, base=10000.0, stream=None):
    """[n, d/2, 2] fp32 (cos, sin) table built by refadapt_rope_axes_table."""
    t = torch.empty((pos.shape[0], int(d) // 2, 2), dtype=torch.float32, device=pos.device)
    refadapt_rope_axes_table(t, pos, axes, base, stream)
    return t


def refadapt_residual_norm(segs, C, post, pre, eps=1e-6, alpha=1.0, mode=None, stream=None):
    """h_out = alpha h + gate N_post(y) post_w; x = N_pre(h_out) pre_w (1 + scale) + shift.
    segs: up to three dicts with h ([B, rows, C] bf16) and, each optional, y,
    h_out, x (the same shape), gate, scale, shift ([B, C] fp32), post_w, pre_w
    ([C] fp32), gated; post, pre: RA_NORM_NONE, RA_NORM_LAYER or RA_NORM_RMS."""
    return check("refadapt_residual_norm", _lib.native().residual_norm(
        segs, int(C), int(post), int(pre), float(eps), float(alpha), mode, _handle(stream)))


def refadapt_residual_norm_backward_workspace_size(B, rows, C) -> int:
    return int(_lib.load().refadapt_residual_norm_backward_workspace_size(int(B), int(rows), int(C)))


def residual_norm_backward_workspace(B, rows, C, device="cuda"):
    """A workspace for refadapt_residual_norm_backward (reusable across calls)."""
    return torch.empty(refadapt_residual_norm_backward_workspace_size(B, rows, C), dtype=torch.uint8, device=device)


def refadapt_residual_norm_backward(seg, C, post, pre, workspace, eps=1e-6, alpha=1.0, err_word=None, stream=None):
    """Gradients of refadapt_residual_norm for one segment: a dict with h (the
    forward call's h_out), y, dx and dh_out (gradients of x and h_out, one may
    be absent), the forward call's gate, scale, post_w, pre_w, and the outputs
    wanted: dh, dy ([B, rows, C] bf16), dgate, dscale, dshift ([B, C] fp32),
    dpost_w, dpre_w ([C] fp32)."""
    return check("refadapt_residual_norm_backward", _lib.native().residual_norm_backward(
        seg, int(C), int(post), int(pre), workspace, float(eps), float(alpha), err_word, _handle(stream)))


def refadapt_glu(segs, F, C, act, mode=None, err_word=None, stream=None):
    """out = act(x w_gate^T) * (x w_up^T). segs: up to three dicts with x ([B,
    rows, C] bf16), w_gate, w_up ([F, C] bf16), out ([B, rows, F] bf16), optional
    pre_gate and pre_up (like out, kept for the backward pass), gated; act:
    RA_ACT_SILU or RA_ACT_GELU. The down projection is refadapt_gemm."""
    return check("refadapt_glu", _lib.native().glu(segs, int(F), int(C), int(act), mode, err_word, _handle(stream)))


def refadapt_glu_backward_workspace_size(B, rows, C, F, O) -> int:
    return int(_lib.load().refadapt_glu_backward_workspace_size(int(B), int(rows), int(C), int(F), int(O)))


def glu_backward_workspace(B, rows, C, F, O, device="cuda"):
    """A workspace for refadapt_glu_backward (reusable across calls)."""
    return torch.empty(refadapt_glu_backward_workspace_size(B, rows, C, F, O), dtype=torch.uint8, device=device)


def refadapt_glu_backward(dy, x, w_gate, w_up, w_down, pre_gate, pre_up, hidden, act, workspace, dx=None, dw_gate=None,
                          dw_up=None, dw_down=None, err_word=None, stream=None):
    """Gradients of y = hidden w_down^T, hidden = act(x w_gate^T) * (x w_up^T), from dy ([B, rows, O] bf16) and what
    refadapt_glu kept (hidden: its out). Fills those of dx ([B, rows, C]), dw_gate, dw_up ([F, C]) and dw_down ([O,
    F]) that are given. x may be None without dw_gate and dw_up, hidden without dw_down."""
    return check("refadapt_glu_backward", _lib.native().glu_backward(
        dy, x, w_gate, w_up, w_down, pre_gate, pre_up, hidden, int(act), workspace, dx, dw_gate, dw_up, dw_down,
        err_word, _handle(stream)))


# --------------------------------------------------------------------------- linear layers in 4 bits
# A weight [N, K] in 4 bits: codes [N, K / 2] and scales (include/refadapt.h has the layout), uint8;
# the scales' exponent and the format (RA_Q4_E4M3 or RA_Q4_E8M0).
Weight4 = collections.namedtuple("Weight4", "codes scales exponent format")


def refadapt_quant4_scales_size(rows, K, format) -> int:
    return int(_lib.load().refadapt_quant4_scales_size(int(rows), int(K), int(format)))


def quant4_buffers(B, rows, C, format, device="cuda"):
    """(codes [B, rows, C / 2], scales [B, row tiles, column tiles, 512]) for refadapt_quant4, uint8."""
    block = 32 if format == RA_Q4_E8M0 else 16
    u8 = dict(dtype=torch.uint8, device=device)
    return (torch.empty((B, rows, C // 2), **u8),
            torch.empty((B, -(-rows // 128), -(-C // (4 * block)), 512), **u8))


def refadapt_quant4(segs, C, format, mode=None, stream=None):
    """bf16 rows to 4 bits. segs: up to three dicts with x ([B, rows, C] bf16) and
    codes ([B, rows, C / 2]) with scales, along the features, or codes_t ([C,
    tokens / 2], tokens = B * rows rounded up to 64) with scales_t, along the rows,
    or both; optional exponent (RA_Q4_E4M3) and gated. Codes and scales are uint8."""
    return check("refadapt_quant4", _lib.native().quant4(segs, int(C), int(format), mode, _handle(stream)))


def weight4(w, format=RA_Q4_E4M3, exponent=None, stream=None):
    """A weight [N, K] bf16 as a Weight4. exponent None: from the weight's largest
    magnitude (which waits for the GPU), so that no scale is cut off and the others have the
    range of e4m3 below it."""
    if w.dim() != 2:
        raise ValueError("w: expected [N, K], got %s" % (tuple(w.shape),))
    if exponent is None:
        exponent = 0
        top = float(w.detach().abs().amax()) if format == RA_Q4_E4M3 and w.numel() else 0.0
        if 0.0 < top < math.inf:
            exponent = min(64, max(-64, math.ceil(math.log2(top / (6.0 * 448.0)))))
    codes, scales = quant4_buffers(1, w.shape[0], w.shape[1], format, w.device)
    refadapt_quant4([{"x": w.detach().unsqueeze(0), "codes": codes, "scales": scales, "exponent": exponent}],
                    w.shape[1], format, stream=stream)
    return Weight4(codes[0], scales[0], exponent, format)


def refadapt_gemm4(segs, N, K, epilogue, format, mode=None, rope=None, H=0, d=0, norm_eps=1e-6, err_word=None,
                   tile_mode=0, stream=None):
    """refadapt_gemm with 4-bit operands. segs: up to three dicts with a ([B, rows,
    K / 2] codes), a_scales, w ([N, K / 2] codes), w_scales, uint8, optional
    a_exponent and w_exponent (RA_Q4_E4M3); the other entries are refadapt_gemm's."""
    return check("refadapt_gemm4", _lib.native().gemm4(
        segs, int(N), int(K), int(epilogue), int(format), mode, rope, int(H), int(d), float(norm_eps), err_word,
        int(tile_mode), _handle(stream)))


def refadapt_linear4_backward_workspace_size(B, rows, K, N) -> int:
    return int(_lib.load().refadapt_linear4_backward_workspace_size(int(B), int(rows), int(K), int(N)))


def linear4_backward_workspace(B, rows, K, N, device="cuda"):
    """A workspace for refadapt_linear4_backward (reusable across calls)."""
    return torch.empty(refadapt_linear4_backward_workspace_size(B, rows, K, N), dtype=torch.uint8, device=device)


def refadapt_linear4_backward(dy, x, w, workspace, dx=None, dw=None, err_word=None, stream=None):
    """Gradients of y = x w^T through 4-bit products (RA_Q4_E8M0), from dy ([B, rows,
    N]), x ([B, rows, K]) and w ([N, K]), bf16. Fills dx ([B, rows, K]) and dw ([N, K])
    where given; x may be None without dw, w without dx."""
    return check("refadapt_linear4_backward", _lib.native().linear4_backward(dy, x, w, workspace, dx, dw, err_word,
                                                                             _handle(stream)))


# --------------------------------------------------------------------------- the optimiser's step
def refadapt_grad_norm_workspace_size() -> int:
    return int(_lib.load().refadapt_grad_norm_workspace_size())


def grad_norm_workspace(device="cuda"):
    """A zero-filled workspace for refadapt_grad_norm (reusable across calls)."""
    return torch.zeros(refadapt_grad_norm_workspace_size(), dtype=torch.uint8, device=device)


def refadapt_grad_norm(grads, max_norm, out, workspace, stream=None):
    """out ([2] fp32) = the norm of all gradients (contiguous fp32 or bf16 tensors)
    together and the factor that clips it to max_norm, for refadapt_adamw's grad_scale."""
    return check("refadapt_grad_norm", _lib.native().grad_norm(grads, float(max_norm), out, workspace,
                                                               _handle(stream)))


def adamw_moments(p, bits=32):
    """Zero moments of a parameter for refadapt_adamw: a dict with m and v, and with
    m_scale and v_scale where bits is 8."""
    if bits == 32:
        return {z: torch.zeros(p.shape, dtype=torch.float32, device=p.device) for z in ("m", "v")}
    if bits != 8:
        raise ValueError("bits: 32 or 8, got %r" % (bits,))
    return {**{z: torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for z in ("m", "v")},
            **{z: torch.ones(-(-p.numel() // 32), dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu)
               for z in ("m_scale", "v_scale")}}


def refadapt_adamw(tensors, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=None, seed=0,
                   stream=None):
    """One AdamW step over all tensors. tensors: a sequence of dicts with p (fp32),
    g (its gradient, fp32 or bf16), m and v (``adamw_moments``: fp32, or e4m3 with
    m_scale and v_scale), optional w (bf16, gets p's rounding). lr and step (from 1
    on): numbers, or fp32 and int32 device tensors of one, which a captured call reads
    when it is replayed. grad_scale: a device tensor of one that the gradients count
    times (not finite: nothing changes). seed: of the 8-bit moments' rounding."""
    return check("refadapt_adamw", _lib.native().adamw(
        tensors, lr, step if isinstance(step, torch.Tensor) else int(step), float(beta1), float(beta2), float(eps),
        float(weight_decay), grad_scale, int(seed), _handle(stream)))
