"""Timed cases of the operators that run and train a DiT block's linear layers in few
bits: products of microscaled 4-bit matrices, and the optimiser's step over all weights
with moments in 32 or 8 bits.

Kinds:

  linear       refadapt_quant4 of the activations, then refadapt_gemm4 with the weights'
               4-bit form, which was made once: what a layer of a block does in a denoising
               step, with the epilogues that the 16-bit product has;
  linear_grad  refadapt_linear4_backward: dx and dw of y = x w^T from dy, x and w in 16 bits,
               through 4-bit products along the features and along the tokens;
  adamw        refadapt_grad_norm and refadapt_adamw: a training step's clipping and update,
               over the tensors of a stack of blocks.

A 4-bit matrix: e2m1 values, two to a byte (the even column in the low half), and one scale
for `block` columns of a row: e4m3 for 16 columns, a power of two (e8m0) for 32; e4m3 scales
stand for their value times 2^exponent, one exponent for the tensor. Scales lie in tiles of
128 rows by 4 blocks, 512 bytes: row r, block j of a tile at 16 (r % 32) + 4 (r / 32) + j.

Values: rows that enter a projection are N(0, 1) (they come out of a norm), weights N(0, 1) /
sqrt(fan_in), gradients 0.01 N(0, 1), AdaLN gates 0.3 + 0.05 N(0, 1). The optimiser's
gradients are 1e-3 N(0, 1), a tensor's times a factor of its own, its moments of that size.
"""
import math

import torch

own = False

MAX_FLOPS = 2.3e12   # of the largest listed call
MAX_BYTES = 9.0e9
E4M3, E8M0 = 0, 1
FORMATS = {"e4m3": E4M3, "e8m0": E8M0}
BLOCK = {E4M3: 16, E8M0: 32}
STORE, GELU, RESID, QKV = 0, 1, 2, 3
EPILOGUES = {"store": STORE, "gelu": GELU, "resid": RESID, "qkv": QKV}
NORM_EPS = 1e-6
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP, SEED, MAX_NORM = 1e-4, 0.9, 0.999, 1e-8, 0.01, 1000, 20240917, 1.0


def listed():
    return [
        # One row: a pooled or conditioning token through an MLP's first layer. Latency
        # and the weights' bytes.
        dict(name="linear_single_row", kind="linear", B=1, text=1, image=0, K=2048, N=8192, epilogue="store",
             format="e4m3"),
        # Ragged text and image rows of three samples, widths that are no power of two.
        dict(name="linear_ragged_gelu", kind="linear", B=3, text=77, image=1209, K=1536, N=6144, epilogue="gelu",
             format="e4m3"),
        # The QKV projection of an image's rows and its prompt: head norms, rotary positions.
        dict(name="linear_qkv", kind="linear", B=1, text=154, image=4096, K=2048, N=6144, epilogue="qkv",
             format="e8m0"),
        # An MLP's second layer: a long K, few columns, the gated residual.
        dict(name="linear_resid_long", kind="linear", B=1, text=512, image=4608, K=8192, N=2048, epilogue="resid",
             format="e4m3"),
        # A video clip's rows through the first layer of a wide block's MLP.
        dict(name="linear_large", kind="linear", B=2, text=0, image=8192, K=4096, N=16384, epilogue="store",
             format="e4m3"),
        # A draft run of an adapter: few rows.
        dict(name="grad_few_rows", kind="linear_grad", B=1, rows=130, K=1024, N=1024),
        # Two images' rows, an odd number of tokens, an MLP's first layer.
        dict(name="grad_image", kind="linear_grad", B=2, rows=1209, K=2048, N=8192),
        # A clip's rows through a square projection.
        dict(name="grad_clip", kind="linear_grad", B=1, rows=16384, K=4096, N=4096),
        # Vectors and small matrices of odd sizes, all that an adapter trains: latency.
        dict(name="adamw_adapter", kind="adamw", layers=2, C=77, F=131, bits=32),
        # A stack of blocks with 32-bit moments.
        dict(name="adamw_stack", kind="adamw", layers=6, C=2048, F=5504, bits=32),
        # One block with 8-bit moments.
        dict(name="adamw8_block", kind="adamw", layers=1, C=1152, F=4608, bits=8),
        # The stack with 8-bit moments.
        dict(name="adamw8_stack", kind="adamw", layers=6, C=2048, F=5504, bits=8),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rows(rng, lo, hi):
    """A row count between lo and hi, odd ones and multiples of 128 among them."""
    n = _log(rng, lo, hi)
    return n // 128 * 128 if n >= 256 and rng.random() < 0.3 else n


def _draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "adamw"])
    if kind == "linear":
        epilogue = rng.choice(list(EPILOGUES))
        K = 64 * _log(rng, 4, 128)
        N = 3 * 256 * _log(rng, 1, 16) if epilogue == "qkv" else 64 * _log(rng, 4, 256)
        return dict(kind=kind, B=rng.choice([1, 1, 2, 3]), text=_rows(rng, 1, 512),
                    image=rng.choice([0, _rows(rng, 16, 8192)]), K=K, N=N, epilogue=epilogue,
                    format=rng.choice(list(FORMATS)))
    if kind == "linear_grad":
        return dict(kind=kind, B=rng.choice([1, 1, 2]), rows=_rows(rng, 1, 8192), K=64 * _log(rng, 4, 96),
                    N=64 * _log(rng, 4, 128))
    return dict(kind=kind, layers=rng.randint(1, 6), C=_log(rng, 16, 2048), F=_log(rng, 16, 5504),
                bits=rng.choice([32, 8]))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return case


# ------------------------------------------------------------------ inputs
def _head_dim(N):
    return 128 if N // 3 % 1024 == 0 else 64


def _streams(case):
    return [(r, case[r]) for r in ("text", "image") if case[r] > 0]


def _to_tiles(s):
    """Scales [..., rows, blocks] in tiles [..., ceil(rows / 128), ceil(blocks / 4), 512], zeros behind the edges."""
    *lead, rows, blocks = s.shape
    t, g = -(-rows // 128), -(-blocks // 4)
    full = s.new_zeros((*lead, t * 128, g * 4))
    full[..., :rows, :blocks] = s
    full = full.view(*lead, t, 4, 32, g, 4).movedim(-2, -4)  # ..., t, g, 4, 32, 4
    return full.transpose(-3, -2).reshape(*lead, t, g, 512).contiguous()


def _from_tiles(s, rows, blocks):
    *lead, t, g, _ = s.shape
    full = s.view(*lead, t, g, 32, 4, 4).transpose(-3, -2).movedim(-4, -2)  # ..., t, 4, 32, g, 4
    return full.reshape(*lead, t * 128, g * 4)[..., :rows, :blocks]


def _blocks_of(x, fmt):
    """x in blocks of its last axis (filled up with zeros), fp32, and each block's scale as 8 bits hold it."""
    b = BLOCK[fmt]
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % b)).unflatten(-1, (-1, b))
    amax = x.abs().amax(-1)
    if fmt == E4M3:
        return x, (amax / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
    e = torch.frexp(amax)[1] - 1                     # amax = mantissa 2^e, mantissa in [1, 2)
    up = (amax > 1.5 * torch.ldexp(torch.ones_like(amax), e)).int()
    byte = torch.where(amax > 0, (e - 2 + up + 127).clamp(min=1), 1).to(torch.uint8)
    return x, byte.view(torch.float8_e8m0fnu)


def _rounded(x, fmt, exponent):
    """The 4-bit values (fp32, in units of their scales) of x and the scales."""
    x, scale = _blocks_of(x * 2.0 ** -exponent, fmt)
    s = scale.float().unsqueeze(-1)
    q = torch.where(s > 0, x / s, 0.0).abs().clamp(max=6.0)
    step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
    return torch.copysign(torch.round(q / step) * step, x), scale


def _quantised(x, fmt, exponent):
    """What x stands for after rounding to 4 bits."""
    q, scale = _rounded(x, fmt, exponent)
    return (q * scale.float().unsqueeze(-1) * 2.0 ** exponent).flatten(-2)[..., :x.shape[-1]]


def _packed(w, fmt, exponent):
    """Codes [N, K / 2] and tiled scales of a weight [N, K]."""
    q, scale = _rounded(w, fmt, exponent)
    grid = torch.tensor(GRID, device=w.device)
    code = torch.bucketize(q.abs(), grid) + 8 * torch.signbit(q)
    code = code.flatten(-2)
    return (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8), _to_tiles(scale.view(torch.uint8))


def _unpacked(codes, scales, fmt, exponent, dtype=torch.float32):
    """The values of a 4-bit weight."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device, dtype=dtype)
    q = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    blocks = -(-q.shape[1] // BLOCK[fmt])
    kind = torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e8m0fnu
    s = _from_tiles(scales, q.shape[0], blocks).contiguous().view(kind).to(dtype)
    return q * s.repeat_interleave(BLOCK[fmt], 1)[:, :q.shape[1]] * 2.0 ** exponent


def _tensors(case):
    """(shapes of matrices, lengths of vectors) of a stack: per layer the QKV, output, gate and up, and down
    projections with their biases and two norms' weights."""
    C, F = case["C"], case["F"]
    return ([(3 * C, C), (C, C), (2 * F, C), (C, F)] * case["layers"], [3 * C, C, 2 * F, C, C, C] * case["layers"])


def _padded(n):
    return -(-n // 32) * 32


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * scale + mean).to(dtype)

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    f32, u8 = torch.float32, torch.uint8
    st = {"case": case}
    if case["kind"] == "linear":
        B, K, N, fmt, epi = case["B"], case["K"], case["N"], FORMATS[case["format"]], EPILOGUES[case["epilogue"]]
        st.update(fmt=fmt, epi=epi, err=torch.zeros(1, dtype=torch.int32, device="cuda"), segs=[])
        d = st["d"] = _head_dim(N) if epi == QKV else 0
        # e4m3 scales of weights of this size are best around one: they are below 2^-6 otherwise
        w_exp = -2 - int(math.ceil(math.log2(K) / 2)) if fmt == E4M3 else 0
        groups = -(-K // (4 * BLOCK[fmt]))
        at = 0
        for _, n in _streams(case):
            w, w_scales = _packed(normal(N, K, scale=K ** -0.5), fmt, w_exp)
            s = {"x": normal(B, n, K), "w": w, "w_scales": w_scales, "w_exp": w_exp, "x_exp": 0,
                 "bias": normal(N, scale=0.05, dtype=f32), "codes": empty(B, n, K // 2, dtype=u8),
                 "scales": empty(B, -(-n // 128), groups, 512, dtype=u8)}
            if epi == QKV:
                H = N // 3 // d
                s.update({z: empty(B, H, n, d) for z in "qkv"}, pos_offset=at,
                         q_norm=normal(d, scale=0.1, mean=1.0, dtype=f32),
                         k_norm=normal(d, scale=0.1, mean=1.0, dtype=f32))
            else:
                s["out"] = empty(B, n, N)
            if epi == RESID:
                s.update(resid=normal(B, n, N), gate=normal(B, N, scale=0.05, mean=0.3, dtype=f32))
            st["segs"].append(s)
            at += n
        if epi == QKV:
            pos = torch.arange(at, device="cuda", dtype=torch.float64)
            ang = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
            st["rope"] = torch.stack((ang.cos(), ang.sin()), -1).float().contiguous()
        return st
    if case["kind"] == "linear_grad":
        B, n, K, N = case["B"], case["rows"], case["K"], case["N"]
        st.update(dy=normal(B, n, N, scale=0.01), x=normal(B, n, K), w=normal(N, K, scale=K ** -0.5),
                  dx=empty(B, n, K), dw=empty(N, K), err=torch.zeros(1, dtype=torch.int32, device="cuda"))
        # A program keeps its scratch from step to step. Its size: codes and scales of dy and x along the
        # tokens, of dy along its features and of w along its outputs, each rounded up to 1 KB.
        def matrix(rows, cols, samples=1):
            return samples * (-(-rows * (cols // 2) // 1024) * 1024 + -(-rows // 128) * -(-cols // 128) * 512 + 1024)
        tokens = -(-B * n // 64) * 64
        st["workspace"] = empty(matrix(N, tokens) + matrix(K, tokens) + B * matrix(n, N) + matrix(K, -(-N // 64) * 64)
                                + (8 << 20), dtype=u8)
        return st
    mats, vecs = _tensors(case)
    total_m, total_v = (sum(map(_padded, ns)) for ns in ([a * b for a, b in mats], vecs))
    factor = torch.rand(len(mats) + len(vecs), generator=g, device="cuda").mul_(4).exp2_().tolist()
    flat = {}
    for part, total in (("m", total_m), ("v", total_v)):
        # the weights' gradients come as the layers' backward passes give them, 16 bits for matrices
        flat["p" + part] = torch.zeros(total, dtype=f32, device="cuda")
        flat["g" + part] = torch.zeros(total, dtype=torch.bfloat16 if part == "m" else f32, device="cuda")
        flat["m" + part] = torch.zeros(total, dtype=f32, device="cuda")
        flat["v" + part] = torch.zeros(total, dtype=f32, device="cuda")
    flat["wm"] = torch.zeros(total_m, dtype=torch.bfloat16, device="cuda")
    places, at = [], {"m": 0, "v": 0}
    for k, shape in enumerate(mats + [(n,) for n in vecs]):
        part, n = "m" if k < len(mats) else "v", math.prod(shape)
        i = at[part]
        size = 1e-3 * factor[k]
        flat["p" + part][i:i + n].normal_(0.0, 0.02, generator=g)
        flat["g" + part][i:i + n].normal_(0.0, size, generator=g)
        flat["m" + part][i:i + n].normal_(0.0, 0.3 * size, generator=g)
        flat["v" + part][i:i + n].uniform_(0.5 * size * size, 1.5 * size * size, generator=g)
        places.append((part, i, n))
        at[part] += _padded(n)
    if case["bits"] == 8:
        for z in "mv":
            for part in "mv":
                q, s = _state8(flat.pop(z + part), None)
                flat[z + part], flat[z + part + "_scale"] = q, s
    st.update(flat=flat, norm=empty(2, dtype=f32), tensors=[], grads=[])
    for part, i, n in places:
        t = {z: flat[z + part][i:i + n] for z in "pgmv"}
        if part == "m":
            t["w"] = flat["wm"][i:i + n]
        if case["bits"] == 8:
            for z in "mv":
                t[z + "_scale"] = flat[z + part + "_scale"][i // 32:i // 32 + _padded(n) // 32]
        st["tensors"].append(t)
        st["grads"].append(t["g"])
    st["workspace"] = torch.zeros(65536, dtype=u8, device="cuda")
    return st


# ------------------------------------------------------------------ the optimiser's 8-bit moments
# Blocks of 32 elements of a tensor, e4m3 values times a power of two (e8m0), the smallest one with
# amax <= 448 2^e. Between two e4m3 values the upper one is taken with the probability that keeps the mean:
# 16 random bits stand for where between them the border lies. A second moment that is not zero is stored as
# the smallest step at least. The random bits of element i (counted over the call's tensors, each from a
# multiple of 32 on) are the halves, low for the first moment, of a 32-bit mix of i, the step and the seed.
def _mix(x):
    mask = 0xffffffff
    x = ((x ^ (x >> 16)) * 0x243f6a89) & mask
    x = ((x ^ (x >> 15)) * 0xb7e15163) & mask
    return x ^ (x >> 16)


def _mix_int(x):
    x = ((x ^ (x >> 16)) * 0x243f6a89) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0xb7e15163) & 0xffffffff
    return x ^ (x >> 16)


def _random_bits(first, n, device):
    """32 bits each for elements first .. first + n (below 2^32) of the call."""
    key = _mix_int(_mix_int(_mix_int(SEED & 0xffffffff) ^ (SEED >> 32)) ^ STEP)
    i = torch.arange(first, first + n, device=device, dtype=torch.int64)
    return _mix(((i * 0x9e3779b1) & 0xffffffff) ^ key)


def _block_scale(x):
    """The e8m0 byte (int32) of each block of 32."""
    amax = x.abs().view(-1, 32).amax(1)
    bits = amax.view(torch.int32)
    return (((bits + 0x1fffff) >> 23) - 8).clamp(1, 254)


def _state8(x, bits16, floor=False):
    """(e4m3 values, e8m0 scales) of a flat fp32 tensor; bits16: random bits, None: to the nearest."""
    byte = _block_scale(x)
    y = (x.view(-1, 32) * ((254 - byte) << 23).view(torch.float32)[:, None]).view(-1)
    if bits16 is None:
        return y.to(torch.float8_e4m3fn), byte.to(torch.uint8).view(torch.float8_e8m0fnu)
    a = y.abs()
    small = a < 2.0 ** -6                      # there the steps are 2^-9, as just above 2^-6
    z = torch.where(small, a + 2.0 ** -6, a)
    z = ((z.view(torch.int32) + (16 * bits16 + 8).int()) & -0x100000).view(torch.float32)
    z = torch.where(small, z - 2.0 ** -6, z)
    if floor:
        z = torch.where(a > 0, z.clamp(min=2.0 ** -9), z)
    return torch.copysign(z, y).to(torch.float8_e4m3fn), byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def _value8(q, scale):
    return (q.float().view(-1, 32) * scale.float()[:, None]).view(-1)


# ------------------------------------------------------------------ the plain forms
def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def _plain_linear(st):
    fmt, epi, outs = st["fmt"], st["epi"], []
    for s in st["segs"]:
        x = _quantised(s["x"], fmt, s["x_exp"])
        y = x @ _unpacked(s["w"], s["w_scales"], fmt, s["w_exp"]).T + s["bias"]
        if epi == GELU:
            y = _gelu(y)
        elif epi == RESID:
            y = s["resid"].float() + s["gate"][:, None] * y
        elif epi == QKV:
            B, n, d = *y.shape[:2], st["d"]
            q, k, v = y.view(B, n, 3, -1, d).permute(2, 0, 3, 1, 4)
            turn = st["rope"][s["pos_offset"]:s["pos_offset"] + n]
            for z, t, w in (("q", q, s["q_norm"]), ("k", k, s["k_norm"])):
                t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + NORM_EPS) * w
                a, b = t[..., 0::2], t[..., 1::2]
                c, sn = turn[..., 0], turn[..., 1]
                outs.append(torch.stack((a * c - b * sn, a * sn + b * c), -1).flatten(-2).bfloat16())
            outs.append(v.bfloat16())
            continue
        outs.append(y.bfloat16())
    return outs


def _plain_linear_grad(st):
    dy, x, w = st["dy"].flatten(0, 1), st["x"].flatten(0, 1), st["w"]
    dx = _quantised(dy, E8M0, 0) @ _quantised(w.T, E8M0, 0).T
    dw = _quantised(dy.T, E8M0, 0) @ _quantised(x.T, E8M0, 0).T
    return [dx.bfloat16().view_as(st["x"]), dw.bfloat16()]


def _plain_adamw(st):
    flat, bits = st["flat"], st["case"]["bits"]
    norm = (flat["gm"].double().square().sum() + flat["gv"].double().square().sum()).sqrt()
    coef = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0).float()
    st["norm"].copy_(torch.stack((norm.float(), coef)))
    bc1, bc2 = 1.0 - BETA1 ** STEP, 1.0 - BETA2 ** STEP
    outs, first = [st["norm"]], 0
    for part in "mv":
        p, g = flat["p" + part], flat["g" + part].float() * coef
        m, v = ((_value8(flat[z + part], flat[z + part + "_scale"]) if bits == 8 else flat[z + part]) for z in "mv")
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * (g * g)
        p.copy_(p - LR * DECAY * p - LR * (m / bc1) / (torch.sqrt(v / bc2) + ADAM_EPS))
        outs.append(p)
        if part == "m":
            outs.append(flat["wm"].copy_(p.bfloat16()))
        if bits == 8:
            r = _random_bits(first, p.numel(), p.device)
            for z, value, b in (("m", m, r & 0xffff), ("v", v, r >> 16)):
                q, s = _state8(value, b, floor=z == "v")
                outs += [flat[z + part].copy_(q), flat[z + part + "_scale"].copy_(s)]
        else:
            outs += [flat["m" + part].copy_(m), flat["v" + part].copy_(v)]
        first += p.numel()
    return outs


# ------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if case["kind"] == "linear":
        if not own:
            return _plain_linear(st)
        from paper_2609_32415_gb300 import api
        K, N, fmt, epi = case["K"], case["N"], st["fmt"], st["epi"]
        api.refadapt_quant4([{"x": s["x"], "codes": s["codes"], "scales": s["scales"], "exponent": s["x_exp"]}
                             for s in st["segs"]], K, fmt)
        segs = []
        for s in st["segs"]:
            t = {"a": s["codes"], "a_scales": s["scales"], "a_exponent": s["x_exp"], "w": s["w"],
                 "w_scales": s["w_scales"], "w_exponent": s["w_exp"], "bias": s["bias"]}
            if epi == QKV:
                t.update(q=s["q"], k=s["k"], v=s["v"], q_norm=s["q_norm"], k_norm=s["k_norm"],
                         pos_offset=s["pos_offset"])
            else:
                t["out"] = s["out"]
            if epi == RESID:
                t.update(resid=s["resid"], gate=s["gate"])
            segs.append(t)
        if epi == QKV:
            api.refadapt_gemm4(segs, N, K, epi, fmt, rope=st["rope"], H=N // 3 // st["d"], d=st["d"],
                               norm_eps=NORM_EPS, err_word=st["err"])
            return [s[z] for s in st["segs"] for z in "qkv"]
        api.refadapt_gemm4(segs, N, K, epi, fmt, err_word=st["err"])
        return [s["out"] for s in st["segs"]]
    if case["kind"] == "linear_grad":
        if not own:
            return _plain_linear_grad(st)
        from paper_2609_32415_gb300 import api
        api.refadapt_linear4_backward(st["dy"], st["x"], st["w"], st["workspace"], dx=st["dx"], dw=st["dw"],
                                      err_word=st["err"])
        return [st["dx"], st["dw"]]
    if not own:
        return _plain_adamw(st)
    from paper_2609_32415_gb300 import api
    api.refadapt_grad_norm(st["grads"], MAX_NORM, st["norm"], st["workspace"])
    api.refadapt_adamw(st["tensors"], LR, STEP, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                       grad_scale=st["norm"][1:], seed=SEED)
    flat, outs = st["flat"], [st["norm"]]
    for part in "mv":
        outs.append(flat["p" + part])
        if part == "m":
            outs.append(flat["wm"])
        for z in "mv":
            outs.append(flat[z + part])
            if case["bits"] == 8:
                outs.append(flat[z + part + "_scale"])
    return outs


def work(case):
    """Bytes: each input read and each output written once. flops: the products'; the optimiser's 15 a weight."""
    if case["kind"] == "linear":
        K, N, nbytes, flops = case["K"], case["N"], 0, 0
        for _, n in _streams(case):
            m = case["B"] * n
            nbytes += 2 * m * K + N * K // 2 + N * K // BLOCK[FORMATS[case["format"]]] + 4 * N + 2 * m * N
            nbytes += 2 * m * N + 4 * case["B"] * N if case["epilogue"] == "resid" else 0
            nbytes += 4 * n * _head_dim(N) if case["epilogue"] == "qkv" else 0
            flops += 2 * m * N * K
        return {"bytes": nbytes, "flops": flops}
    if case["kind"] == "linear_grad":
        m, K, N = case["B"] * case["rows"], case["K"], case["N"]
        return {"bytes": 2 * (m * N + 2 * m * K + 2 * N * K), "flops": 4 * m * N * K}
    mats, vecs = _tensors(case)
    n, k = sum(a * b for a, b in mats), sum(vecs)
    states = 16 if case["bits"] == 32 else 4.125
    return {"bytes": n * (8 + 2 + 2 + states) + k * (8 + 4 + states), "flops": 15 * (n + k)}


# ------------------------------------------------------------------ 64 bits
def _nearest4(x, fmt, exponent):
    """The values of x in 4 bits, in 64 bits, by distance to the grid."""
    b, K = BLOCK[fmt], x.shape[-1]
    v = x.double() * 2.0 ** -exponent
    v = torch.cat((v, v.new_zeros((*v.shape[:-1], -K % b))), -1)
    v = v.view(*v.shape[:-1], -1, b)
    top = v.abs().max(-1, keepdim=True).values
    if fmt == E4M3:
        # e4m3: 3 bits behind the leading one, steps of 2^-9 below 2^-6, at most 448
        t = (top / 6).clamp(max=448.0)
        step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
        s = torch.round(t / step) * step
    else:
        s = torch.exp2(torch.ceil(torch.log2((top / 6).clamp(min=2.0 ** -126))))
        s = torch.where(top > 6 * s, 2 * s, torch.where(top <= 3 * s, s / 2, s)).clamp(min=2.0 ** -126)
    grid = torch.tensor(GRID, device=x.device, dtype=torch.float64)
    near = torch.zeros_like(v)
    a = v.abs()
    for lo, hi, even in zip(GRID[:-1], GRID[1:], (True, False) * 4):  # the even code takes the middle
        mid = 0.5 * (lo + hi) * s
        near = torch.where((a > mid) | ((a == mid) & (not even)), grid.new_tensor(hi), near)
    return (torch.copysign(near, v) * s * 2.0 ** exponent).flatten(-2)[..., :K]


def exact(case, seed):
    if work(case)["flops"] > MAX_FLOPS:
        return None
    st = prepare(case, seed)
    if case["kind"] == "linear":
        outs = []
        for s in st["segs"]:
            w = _unpacked(s["w"], s["w_scales"], st["fmt"], s["w_exp"], torch.float64)
            y = torch.matmul(_nearest4(s["x"], st["fmt"], s["x_exp"]), w.T).add_(s["bias"].double())
            if st["epi"] == GELU:
                y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
            elif st["epi"] == RESID:
                y = y * s["gate"].double().unsqueeze(1) + s["resid"].double()
            elif st["epi"] == QKV:
                B, n, d = y.shape[0], y.shape[1], st["d"]
                parts = y.view(B, n, 3, -1, d).transpose(1, 3)  # B, H, 3, n, d
                turn = torch.view_as_complex(st["rope"][s["pos_offset"]:s["pos_offset"] + n].double())
                for i, w in ((0, s["q_norm"]), (1, s["k_norm"])):
                    t = parts[:, :, i]
                    t = t / (t.pow(2).sum(-1, keepdim=True) / d + NORM_EPS).sqrt() * w.double()
                    z = torch.view_as_complex(t.contiguous().view(*t.shape[:-1], d // 2, 2)) * turn
                    outs.append(torch.view_as_real(z).flatten(-2))
                outs.append(parts[:, :, 2])
                continue
            outs.append(y)
        return outs
    if case["kind"] == "linear_grad":
        dy, x = st["dy"].flatten(0, 1), st["x"].flatten(0, 1)
        dx = torch.matmul(_nearest4(dy, E8M0, 0), _nearest4(st["w"].T, E8M0, 0).T)
        dw = torch.matmul(_nearest4(dy.T, E8M0, 0), _nearest4(x.T, E8M0, 0).T)
        return [dx.view(st["x"].shape), dw]
    flat, bits, first = st["flat"], case["bits"], 0
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(flat["g" + z].double()) for z in "mv"]))
    coef = (MAX_NORM / norm).clamp(max=1.0)
    outs = [torch.stack((norm, coef))]
    for part in "mv":
        n = flat["p" + part].numel()
        g = flat["g" + part].double().mul_(coef)
        state = []
        for z in "mv":
            s = flat[z + part].double()
            state.append(s.view(-1, 32).mul_(flat[z + part + "_scale"].double().unsqueeze(1)).view(-1) if bits == 8
                         else s)
        m = state[0].mul_(BETA1).add_(g, alpha=1.0 - BETA1)
        v = state[1].mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
        del g, state
        p = flat["p" + part].double() * (1.0 - LR * DECAY)
        p -= LR * (m / (1.0 - BETA1 ** STEP)) / ((v / (1.0 - BETA2 ** STEP)).sqrt() + ADAM_EPS)
        outs.append(p)
        if part == "m":
            outs.append(p)
        r = _random_bits(first, n, p.device) if bits == 8 else None
        for z, value in (("m", m), ("v", v)):
            if bits == 32:
                outs.append(value)
                continue
            top = value.abs().view(-1, 32).amax(1)
            s = torch.exp2(torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -126))))
            s = torch.where(top > 448 * s, 2 * s, torch.where(top <= 224 * s, s / 2, s)).clamp(min=2.0 ** -126)
            y = (value.view(-1, 32) / s.unsqueeze(1)).view(-1)
            a = y.abs()
            step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
            low = torch.floor(a / step)
            border = ((r & 0xffff if z == "m" else r >> 16).double() * 16 + 8) / 2.0 ** 20
            q = (low + (a / step - low + border >= 1.0)) * step
            q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q) if z == "v" else q
            outs += [torch.copysign(q, y), s]
        first += n
    return outs
