"""refadapt_quant4, refadapt_gemm4 and refadapt_linear4_backward against fp64.

Quantisation is exact: codes and scales equal the oracle's. A product's operands are exact
and their products too (2 + 2 significant bits of codes, 4 + 4 of scales), so what differs
from fp64 is the sum of K terms in fp32, in any order and with partial sums that may be cut
off instead of rounded: at most K 2^-23 sum |a w|; and one rounding of the output, half a
step of bf16, 2^-8 of the value. Epilogues are fp32: a few 2^-24 of their operands, covered
by 2^-20 of the magnitudes that enter."""
import numpy as np
import pytest
import torch

from _helpers import f64
from oracle import lowbit

pytestmark = pytest.mark.gpu

STORE, GELU, RESID, QKV = 0, 1, 2, 3
E4M3, E8M0 = lowbit.E4M3, lowbit.E8M0
BF, F32 = 2.0 ** -8, 2.0 ** -20


def api():
    from paper_2609_32415_gb300 import api as a
    return a


def bf(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).cuda()


def filled(shape, fill=0xa5):
    return torch.full(shape, fill, dtype=torch.uint8, device="cuda")


def quantised(x, fmt, exponent=0):
    """The call's (codes, scales) of [B, rows, C]."""
    a = api()
    codes, scales = a.quant4_buffers(*x.shape, fmt)
    a.refadapt_quant4([{"x": x, "codes": codes, "scales": scales, "exponent": exponent}], x.shape[2], fmt)
    return codes, scales


def check_rows(x, codes, scales, fmt, exponent=0):
    for s in range(x.shape[0]):
        want, byte = lowbit.quantise(f64(x[s]), fmt, exponent)
        fine = np.isfinite(np.abs(f64(x[s])).reshape(x.shape[1], -1, lowbit.BLOCK[fmt]).max(-1))
        got = codes[s].cpu().numpy()
        mask = np.repeat(fine, lowbit.BLOCK[fmt] // 2, 1)  # codes under a NaN scale say nothing
        assert np.array_equal(got[mask], lowbit.pack(want)[mask])
        assert np.array_equal(scales[s].cpu().numpy(), lowbit.tiles(byte))


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("B, rows, C", [(1, 1, 64), (2, 3, 192), (1, 127, 256), (3, 129, 320), (1, 300, 1088)])
def test_rows_are_exact(cuda_ok, fmt, B, rows, C):
    g = torch.Generator().manual_seed(rows + C)
    # magnitudes over many binades, so that scales of every kind occur
    x = (torch.randn((B, rows, C), generator=g) * 2.0 ** torch.randint(-14, 12, (B, rows, 1), generator=g)).bfloat16().cuda()
    codes, scales = quantised(x, fmt)
    check_rows(x, codes, scales, fmt)


@pytest.mark.parametrize("exponent", [-64, -9, 3, 64])
def test_rows_with_an_exponent(cuda_ok, exponent):
    g = torch.Generator().manual_seed(exponent + 100)
    x = bf((1, 40, 128), g, 2.0 ** exponent)
    codes, scales = quantised(x, E4M3, exponent)
    check_rows(x, codes, scales, E4M3, exponent)


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
def test_every_border_and_extreme(cuda_ok, fmt):
    """Quotients that are exactly between two values, for every scale; zeros, the smallest and largest bf16."""
    block = lowbit.BLOCK[fmt]
    edges = np.array([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.0])
    edges = np.concatenate([edges, -edges])[:block] if block == 32 else edges
    rows = []
    for byte in range(1, 127):
        s = lowbit.E4M3_VALUES[byte] if fmt == E4M3 else 2.0 ** (byte - 100.0)
        rows.append(np.tile(edges * s, 64 // block))
    for big in (0.0, 1e-38, 2.0 ** -133, 2.0 ** -126, 3.3895e38, -3.3895e38, 2688.0, 2752.0, 3000.0):
        r = np.zeros(64)
        r[5], r[40] = big, big / 3
        rows.append(r)
    x = torch.tensor(np.array(rows), dtype=torch.float32).bfloat16().cuda()[None]
    codes, scales = quantised(x, fmt)
    check_rows(x, codes, scales, fmt)


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite(cuda_ok, fmt, bad):
    """Their block's scale is NaN, the other blocks are as without them."""
    g = torch.Generator().manual_seed(3)
    x = bf((1, 5, 128), g)
    x[0, 2, 37] = bad
    codes, scales = quantised(x, fmt)
    check_rows(x, codes, scales, fmt)


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("B, rows, C", [(1, 1, 8), (1, 64, 64), (2, 37, 72), (3, 129, 200), (1, 257, 128)])
@pytest.mark.parametrize("both", [False, True])
def test_along_the_rows(cuda_ok, fmt, B, rows, C, both):
    if both and C % 64:
        C = 64 * (C // 64 + 1)
    a, g = api(), torch.Generator().manual_seed(C)
    x = (torch.randn((B, rows, C), generator=g) * 2.0 ** torch.randint(-6, 6, (1, 1, C), generator=g)).bfloat16().cuda()
    tokens = -(-B * rows // 64) * 64
    seg = {"x": x, "codes_t": filled((C, tokens // 2)),
           "scales_t": filled((a.refadapt_quant4_scales_size(C, tokens, fmt),))}
    if both:
        seg["codes"], seg["scales"] = filled((B, rows, C // 2)), filled((B * a.refadapt_quant4_scales_size(rows, C, fmt),))
    a.refadapt_quant4([seg], C, fmt)
    xt = np.zeros((C, tokens))
    xt[:, :B * rows] = f64(x.reshape(-1, C)).T
    want, byte = lowbit.quantise(xt, fmt)
    assert np.array_equal(seg["codes_t"].cpu().numpy(), lowbit.pack(want))
    assert np.array_equal(seg["scales_t"].cpu().numpy(), lowbit.tiles(byte).reshape(-1))
    if both:
        check_rows(x, seg["codes"], seg["scales"].view(B, -1, -(-C // (4 * lowbit.BLOCK[fmt])), 512), fmt)


def test_rows_with_strides_segments_and_gates(cuda_ok):
    """Two segments in one call: one in a wider buffer, one gated for a sample that reuses."""
    a, g = api(), torch.Generator().manual_seed(9)
    wide = bf((2, 50, 256), g)
    x, y = wide[:, :33, 64:192], bf((2, 20, 128), g)
    codes = filled((2, 40, 96))
    segs = [{"x": x, "codes": codes[:, :33, 16:80], "scales": filled((2, 1, 2, 512))},
            {"x": y, "codes": filled((2, 20, 64)), "scales": filled((2, 1, 2, 512)), "gated": True}]
    a.refadapt_quant4(segs, 128, E4M3, mode=torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    check_rows(x, segs[0]["codes"], segs[0]["scales"], E4M3)
    assert bool((codes[:, 33:] == 0xa5).all()) and bool((codes[:, :33, :16] == 0xa5).all())
    assert bool((segs[1]["codes"][0] == 0xa5).all()) and bool((segs[1]["scales"][0] == 0xa5).all())
    check_rows(y[1:], segs[1]["codes"][1:], segs[1]["scales"][1:], E4M3)


def test_weight4_takes_the_whole_range(cuda_ok):
    a, g = api(), torch.Generator().manual_seed(11)
    w = bf((128, 256), g, 2.0 ** -20)
    q = a.weight4(w)
    byte = lowbit.untile(q.scales.cpu().numpy(), 128, 16)
    top = float(w.abs().max()) / 6 / 2.0 ** q.exponent
    assert 224 < top <= 448 and byte.max() <= 126
    codes, scales = quantised(w[None], E4M3, q.exponent)
    assert torch.equal(codes[0], q.codes) and torch.equal(scales[0], q.scales)
    assert a.weight4(torch.zeros((64, 64), dtype=torch.bfloat16, device="cuda")).exponent == 0


# ------------------------------------------------------------------ products
def values_of(codes, scales, fmt, exponent=0):
    """[rows, K] fp64 of one matrix's codes and scales."""
    c = codes.cpu().numpy()
    full = np.zeros((c.shape[0], 2 * c.shape[1]), np.int64)
    full[:, 0::2], full[:, 1::2] = c & 15, c >> 4
    byte = lowbit.untile(scales.cpu().numpy(), c.shape[0], -(-full.shape[1] // lowbit.BLOCK[fmt]))
    return lowbit.values(full, byte, fmt, exponent)


def operands(B, rows, N, K, fmt, g, a_exp=0, w_exp=0):
    x, w = bf((B, rows, K), g, 2.0 ** a_exp), bf((N, K), g, K ** -0.5)
    codes, scales = quantised(x, fmt, a_exp)
    wc, ws = quantised(w[None], fmt, w_exp)
    wc, ws = wc[0], ws[0]
    aw = [values_of(codes[s], scales[s], fmt, a_exp) for s in range(B)]
    wv = values_of(wc, ws, fmt, w_exp)
    seg = {"a": codes, "a_scales": scales, "a_exponent": a_exp, "w": wc, "w_scales": ws, "w_exponent": w_exp}
    return seg, np.stack([v @ wv.T for v in aw]), np.stack([np.abs(v) @ np.abs(wv).T for v in aw]) * K * 2.0 ** -23


def gelu64(x):
    return x / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)))


def within(got, ref, tol):
    got = f64(got)
    assert np.isfinite(got).all()
    worst = float(np.max(np.abs(got - ref) / tol))
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 64, 64), (2, 3, 192, 128), (1, 127, 256, 320), (1, 128, 448, 256), (2, 129, 320, 576),
          (1, 300, 1024, 1088), (1, 517, 640, 2048)]


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("tile_mode", [0, 1, 2])
@pytest.mark.parametrize("B, rows, N, K", SHAPES)
def test_product(cuda_ok, fmt, tile_mode, B, rows, N, K):
    g = torch.Generator().manual_seed(rows + N)
    exps = (2, -6) if fmt == E4M3 else (0, 0)
    seg, y, acc = operands(B, rows, N, K, fmt, g, *exps)
    bias = (0.3 * torch.randn(N, generator=g)).cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    guard = torch.full((B, rows + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    seg.update(bias=bias, out=guard[:, :rows])
    api().refadapt_gemm4([seg], N, K, STORE, fmt, tile_mode=tile_mode, err_word=err)
    ref = y + f64_32(bias)
    within(seg["out"], ref, BF * np.abs(ref) + acc + F32 * (np.abs(y) + np.abs(ref)) + 1e-30)
    assert bool((guard[:, rows:] == 7.0).all()) and int(err) == 0


def f64_32(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("epilogue", [GELU, RESID])
@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("tile_mode", [1, 2])
def test_epilogues_of_two_segments(cuda_ok, epilogue, fmt, tile_mode):
    """Text and image rows with weights of their own; the residual in place for one of them."""
    g = torch.Generator().manual_seed(17 + epilogue)
    B, N, K = 2, 320, 448
    segs, refs = [], []
    for rows in (33, 260):
        seg, y, acc = operands(B, rows, N, K, fmt, g)
        seg["bias"] = (0.3 * torch.randn(N, generator=g)).cuda()
        seg["out"] = torch.empty((B, rows, N), dtype=torch.bfloat16, device="cuda")
        x = y + f64_32(seg["bias"])
        if epilogue == GELU:
            ref = gelu64(x)
            tol = BF * np.abs(ref) + 1.2 * acc + 16 * F32 * (np.abs(x) + np.abs(y))
        else:
            seg["gate"] = torch.randn((B, N), generator=g).cuda()
            seg["resid"] = bf((B, rows, N), g)
            gate = f64_32(seg["gate"])[:, None]
            ref = f64(seg["resid"]) + gate * x
            tol = BF * np.abs(ref) + np.abs(gate) * (acc + F32 * (np.abs(x) + np.abs(y))) + F32 * np.abs(ref)
            if rows == 33:
                seg["out"] = seg["resid"]
        segs.append(seg)
        refs.append((ref, tol + 1e-30))
    api().refadapt_gemm4(segs, N, K, epilogue, fmt, tile_mode=tile_mode)
    for seg, (ref, tol) in zip(segs, refs):
        within(seg["out"], ref, tol)


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("epilogue", [STORE, GELU, RESID])
@pytest.mark.parametrize("B, rows, N, K, mode", [(1, 1, 64, 64, 0), (1, 1, 192, 1088, 2), (1, 1, 448, 2048, 2), (1, 1, 320, 1024, 1),
                                                 (1, 1, 128, 4160, 2), (1, 1, 64, 8192, 0), (2, 1, 256, 128, 2),
                                                 (1, 3, 448, 2048, 2)])
def test_few_rows(cuda_ok, fmt, epilogue, B, rows, N, K, mode):
    """One row goes to a kernel of its own: two segments, the second gated; the tensor cores' result beside it
    (tile_mode 1) is within the same bound, as are those of a few rows."""
    a, g = api(), torch.Generator().manual_seed(N + K + epilogue)
    mode = torch.tensor([mode, 0][:B], dtype=torch.int32, device="cuda")
    segs, want = [], []
    for gated in (False, True):
        seg, y, acc = operands(B, rows, N, K, fmt, g, *((1, -5) if fmt == E4M3 else (0, 0)))
        seg.update(gated=gated, bias=(0.3 * torch.randn(N, generator=g)).cuda() if not gated else None)
        seg["out"] = torch.full((B, rows, N + 8), 7.0, dtype=torch.bfloat16, device="cuda")[..., :N]
        x = y + (f64_32(seg["bias"]) if not gated else 0.0)
        if epilogue == STORE:
            ref, tol = x, acc
        elif epilogue == GELU:
            ref, tol = gelu64(x), 1.2 * acc + 16 * F32 * np.abs(x)
        else:
            seg.update(gate=torch.randn((B, N), generator=g).cuda(), resid=bf((B, rows, N), g))
            gate = f64_32(seg["gate"])[:, None]
            ref, tol = f64(seg["resid"]) + gate * x, np.abs(gate) * acc
        segs.append(seg)
        want.append((ref, tol + BF * np.abs(ref) + 4 * F32 * (np.abs(x) + np.abs(ref)) + 1e-30))
    for tile_mode in (0, 1):
        a.refadapt_gemm4(segs, N, K, epilogue, fmt, mode=mode, tile_mode=tile_mode)
        assert ("one row" in a.refadapt_last_launch()) == (tile_mode == 0 and B * rows == 1)
        for seg, (ref, tol) in zip(segs, want):
            for s in range(B):
                if seg["gated"] and int(mode[s]) == 0:
                    assert bool((seg["out"][s] == 7.0).all())
                else:
                    within(seg["out"][s], ref[s], tol[s])
        for seg in segs:
            seg["out"].fill_(7.0)


def test_one_row_of_every_code_and_scale(cuda_ok):
    """Every code and scale byte, NaN ones among them, as the tensor cores have it."""
    a, N, K = api(), 1024, 512
    g = torch.Generator().manual_seed(5)
    for fmt in (E4M3, E8M0):
        codes, w = (torch.randint(0, 256, s, generator=g, dtype=torch.uint8).cuda() for s in ((1, 1, K // 2), (N, K // 2)))
        sizes = [a.refadapt_quant4_scales_size(r, K, fmt) for r in (1, N)]
        lo, hi = (0, 128) if fmt == E4M3 else (120, 134)
        scales = [torch.randint(lo, hi, (n,), generator=g, dtype=torch.uint8).cuda() for n in sizes]
        scales[1][::97] = 0x7f if fmt == E4M3 else 0xff
        outs = []
        for tile_mode in (0, 1):
            out = torch.empty((1, 1, N), dtype=torch.bfloat16, device="cuda")
            a.refadapt_gemm4([{"a": codes, "a_scales": scales[0], "w": w, "w_scales": scales[1], "out": out}], N, K, STORE, fmt,
                             tile_mode=tile_mode)
            outs.append(out.float())
        nan = [torch.isnan(o) for o in outs]
        assert torch.equal(*nan) and bool(nan[0].any()) and not bool(nan[0].all())
        rel = (outs[0] - outs[1])[~nan[0]].norm() / outs[1][~nan[0]].norm()
        assert float(rel) < BF  # both within half a bf16 step of sums that differ by far less


@pytest.mark.parametrize("H, d", [(4, 64), (2, 128), (6, 128)])
@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("tile_mode", [1, 2])
def test_qkv(cuda_ok, H, d, fmt, tile_mode):
    """Head norms, rotary positions, v; two segments, the second gated: sample 0 reuses (nothing is
    written), sample 1 at the boundary (its query only), sample 2 in full."""
    a, g = api(), torch.Generator().manual_seed(H)
    B, K, eps = 3, 256, 1e-6
    C = H * d
    rope = a.rope_table(400, d)
    mode = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    segs, want = [], []
    for rows, at, gated in ((20, 0, False), (150, 20, True)):
        seg, y, acc = operands(B, rows, 3 * C, K, fmt, g)
        seg["bias"] = (0.3 * torch.randn(3 * C, generator=g)).cuda()
        for z in "qkv":
            seg[z] = torch.full((B, H, rows, d), 7.0, dtype=torch.bfloat16, device="cuda")
        seg.update(q_norm=(1 + 0.1 * torch.randn(d, generator=g)).cuda(), pos_offset=at, gated=gated,
                   k_norm=(1 + 0.1 * torch.randn(d, generator=g)).cuda())
        x = (y + f64_32(seg["bias"])).reshape(B, rows, 3, H, d).transpose(2, 0, 3, 1, 4)
        e = (acc + F32 * np.abs(y)).reshape(B, rows, 3, H, d).transpose(2, 0, 3, 1, 4)
        table = f64_32(rope)[at:at + rows]
        for i, z in enumerate("qkv"):
            if z == "v":
                ref, tol = x[i], BF * np.abs(x[i]) + e[i]
            else:
                rms = np.sqrt((x[i] ** 2).mean(-1, keepdims=True) + eps)
                w = f64_32(seg[z + "_norm"])
                n = x[i] / rms * w
                c, s = table[..., 0], table[..., 1]
                ref = np.empty_like(n)
                ref[..., 0::2] = n[..., 0::2] * c - n[..., 1::2] * s
                ref[..., 1::2] = n[..., 0::2] * s + n[..., 1::2] * c
                # the error of x in both of a pair, and through the norm (at most the mean error times n)
                ex = e[i].max(-1, keepdims=True) / rms
                tol = BF * np.abs(ref) + 2 * ex * (np.abs(w).max() + np.abs(n).max(-1, keepdims=True)) + \
                    4 * F32 * np.abs(n).max(-1, keepdims=True)
            want.append((seg, z, ref, tol + 1e-30, gated))
        segs.append(seg)
    a.refadapt_gemm4(segs, 3 * C, K, QKV, fmt, mode=mode, rope=rope, H=H, d=d, norm_eps=eps, tile_mode=tile_mode)
    for seg, z, ref, tol, gated in want:
        for s in range(B):
            if gated and (s == 0 or (s == 1 and z != "q")):
                assert bool((seg[z][s] == 7.0).all())
            else:
                within(seg[z][s], ref[s], tol[s])


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
@pytest.mark.parametrize("epilogue, tile_mode, N, d",
                         [(e, *case, 0) for e in (STORE, GELU, RESID)
                          for case in ((1, 64), (1, 128), (1, 320), (2, 64), (2, 128), (2, 192), (2, 448))] +
                         [(QKV, t, 768, d) for t in (1, 2) for d in (64, 128)])
def test_many_tiles(cuda_ok, fmt, epilogue, tile_mode, N, d):
    """Several tiles to a CTA, with one to three units of columns: every row has what the same row has in a
    call of one tile to a CTA (the sums' order is the same), whose values other tests check."""
    a, g = api(), torch.Generator().manual_seed(N + epilogue)
    few, rows, K = 301, 128 * 152 * 3 + 77, 192
    base, w = bf((1, few, K), g), bf((N, K), g) * 0.1
    wc, ws = (t[0] for t in quantised(w[None].to(torch.bfloat16), fmt))
    at = (torch.arange(rows, device="cuda") * 7) % few
    resid, gate, bias = bf((1, few, N), g), torch.randn((1, N), generator=g).cuda(), torch.randn(N, generator=g).cuda()

    def run(x, res):
        codes, scales = quantised(x, fmt)
        n = x.shape[1]
        seg = {"a": codes, "a_scales": scales, "w": wc, "w_scales": ws, "bias": bias}
        kw = {}
        if epilogue == QKV:
            H = N // 3 // d
            outs = [torch.empty((1, H, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
            norm = torch.linspace(0.5, 1.5, d, device="cuda")
            seg.update(q=outs[0], k=outs[1], v=outs[2], q_norm=norm, k_norm=norm, pos_offset=0)
            kw = dict(rope=a.rope_table(5, d)[4:].expand(n, -1, -1).contiguous(), H=H, d=d)
        else:
            outs = [torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda")]
            seg["out"] = outs[0]
            if epilogue == RESID:
                seg.update(resid=res, gate=gate)
        a.refadapt_gemm4([seg], N, K, epilogue, fmt, tile_mode=tile_mode, **kw)
        return torch.cat(outs, 1) if epilogue == QKV else outs[0]

    want = run(base, resid)
    got = run(base[:, at].contiguous(), resid[:, at].contiguous())
    assert torch.equal(got, want[..., at, :])


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
def test_long_call_after_short(cuda_ok, fmt):
    """Long calls keep more of their operands on the way than short ones do, which came first here."""
    a, g = api(), torch.Generator().manual_seed(41)
    rows, N, K = 8192, 8192, 8192
    x, w = bf((1, rows, K), g), bf((1, N, K), g)
    wc, ws = (t[0] for t in quantised(w, fmt))
    outs = []
    for n in (256, rows):
        codes, scales = quantised(x[:, :n].contiguous(), fmt)
        out = torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda")
        a.refadapt_gemm4([{"a": codes, "a_scales": scales, "w": wc, "w_scales": ws, "out": out}], N, K, STORE, fmt, tile_mode=2)
        outs.append(out)
    assert torch.equal(outs[1][:, :256], outs[0])
    a.refadapt_gemm4([{"a": codes[:, :256].contiguous(), "a_scales": scales[:, :2].contiguous(), "w": wc, "w_scales": ws,
                       "out": outs[0].zero_()}], N, K, STORE, fmt, tile_mode=2)
    assert torch.equal(outs[1][:, :256], outs[0])


def test_product_of_no_rows_and_nan_rows(cuda_ok):
    """A segment without rows is skipped; a row with a NaN scale is NaN and no other one."""
    g = torch.Generator().manual_seed(23)
    N, K = 128, 128
    seg, y, acc = operands(1, 40, N, K, E4M3, g)
    x = bf((1, 40, K), g)
    x[0, 7, 3] = float("nan")
    seg["a"], seg["a_scales"] = quantised(x, E4M3)
    seg["out"] = torch.zeros((1, 40, N), dtype=torch.bfloat16, device="cuda")
    empty = {"a": filled((1, 0, K // 2)), "a_scales": filled((1, 0, 2, 512)), "w": seg["w"], "w_scales": seg["w_scales"],
             "out": torch.empty((1, 0, N), dtype=torch.bfloat16, device="cuda")}
    api().refadapt_gemm4([empty, seg], N, K, STORE, E4M3)
    nan = torch.isnan(seg["out"][0]).all(1)
    assert bool(nan[7]) and int(torch.isnan(seg["out"]).any(-1).sum()) == 1


def test_product_is_the_same_in_a_graph_and_twice(cuda_ok):
    g = torch.Generator().manual_seed(29)
    a = api()
    x, N, K = bf((2, 200, 512), g), 576, 512
    w = a.weight4(bf((N, K), g, K ** -0.5), E8M0)
    codes, scales = a.quant4_buffers(2, 200, K, E8M0)
    out = torch.empty((2, 200, N), dtype=torch.bfloat16, device="cuda")

    def layer():
        a.refadapt_quant4([{"x": x, "codes": codes, "scales": scales}], K, E8M0)
        a.refadapt_gemm4([{"a": codes, "a_scales": scales, "w": w.codes, "w_scales": w.scales, "out": out}], N, K, STORE,
                         E8M0)

    layer()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        layer()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    x.mul_(2)  # the replay reads what is there: powers of two scale exactly
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.float(), first.float() * 2)


# ------------------------------------------------------------------ gradients
@pytest.mark.parametrize("B, rows, K, N", [(1, 1, 64, 64), (2, 37, 192, 128), (1, 130, 320, 448), (3, 129, 256, 640)])
@pytest.mark.parametrize("wanted", ["both", "dx", "dw"])
def test_gradients(cuda_ok, B, rows, K, N, wanted):
    a, g = api(), torch.Generator().manual_seed(K + N + rows)
    dy, x, w = bf((B, rows, N), g, 0.01), bf((B, rows, K), g), bf((N, K), g, K ** -0.5)
    ws = a.linear4_backward_workspace(B, rows, K, N)
    ws.fill_(0xa5)
    dx = torch.empty((B, rows, K), dtype=torch.bfloat16, device="cuda") if wanted != "dw" else None
    dw = torch.empty((N, K), dtype=torch.bfloat16, device="cuda") if wanted != "dx" else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    a.refadapt_linear4_backward(dy, x if dw is not None else None, w if dx is not None else None, ws, dx=dx, dw=dw,
                                err_word=err)
    y64, x64, w64 = f64(dy.reshape(-1, N)), f64(x.reshape(-1, K)), f64(w)
    assert int(err) == 0
    if dx is not None:
        p, q = lowbit.rounded(y64, E8M0), lowbit.rounded(w64.T, E8M0)
        ref = p @ q.T
        within(dx.reshape(-1, K), ref, BF * np.abs(ref) + N * 2.0 ** -23 * (np.abs(p) @ np.abs(q).T) + 1e-30)
    if dw is not None:
        p, q = lowbit.rounded(y64.T, E8M0), lowbit.rounded(x64.T, E8M0)
        ref = p @ q.T
        within(dw, ref, BF * np.abs(ref) + (B * rows + 64) * 2.0 ** -23 * (np.abs(p) @ np.abs(q).T) + 1e-30)


@pytest.mark.parametrize("B, rows, K, N", [(1, 130, 1024, 1024), (2, 1209, 2048, 8192), (1, 5000, 1024, 4096), (1, 300, 4096, 64),
                                           (1, 7000, 64, 192), (3, 700, 3008, 2048)])
def test_gradients_together_are_those_alone(cuda_ok, B, rows, K, N):
    """Both products of a call share a launch, whose CTAs take unlike numbers of their tiles."""
    a, g = api(), torch.Generator().manual_seed(rows)
    dy, x, w = bf((B, rows, N), g, 0.01), bf((B, rows, K), g), bf((N, K), g, K ** -0.5)
    ws = a.linear4_backward_workspace(B, rows, K, N)
    both = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    a.refadapt_linear4_backward(dy, x, w, ws, dx=both[0], dw=both[1])
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    a.refadapt_linear4_backward(dy, x, w, ws, dx=dx)
    a.refadapt_linear4_backward(dy, x, w, ws, dw=dw)
    assert torch.equal(both[0], dx) and torch.equal(both[1], dw)


def test_gradients_without_rows(cuda_ok):
    a = api()
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    dw = torch.ones((64, 128), dtype=torch.bfloat16, device="cuda")
    a.refadapt_linear4_backward(e(2, 0, 64), e(2, 0, 128), e(64, 128), a.linear4_backward_workspace(2, 0, 128, 64),
                                dx=e(2, 0, 128), dw=dw)
    assert bool((dw == 0).all())


def test_gradients_of_strided_rows(cuda_ok):
    """dy and x as parts of wider buffers; the same bits as of whole ones."""
    a, g = api(), torch.Generator().manual_seed(41)
    B, rows, K, N = 2, 50, 128, 192
    dy, x, w = bf((B, rows + 5, N + 64), g, 0.01)[:, 2:2 + rows, :N], bf((B, rows + 1, K + 8), g)[:, :rows, 8:], bf((N, K), g)

    def grads(dy, x):
        dx, dw = torch.empty((B, rows, K), dtype=torch.bfloat16, device="cuda"), torch.empty_like(w)
        a.refadapt_linear4_backward(dy, x, w, a.linear4_backward_workspace(B, rows, K, N), dx=dx, dw=dw)
        return dx, dw

    for s, t in zip(grads(dy, x), grads(dy.contiguous(), x.contiguous())):
        assert torch.equal(s, t)
