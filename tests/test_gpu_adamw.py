"""refadapt_grad_norm and refadapt_adamw against fp64.

Tolerances. fp32 moments: two products and a sum, each rounded: 3 half steps of fp32 (2^-24
each) of the terms' magnitudes, one more for the betas as fp32 and one for the clipped gradient:
2^-21 in all of sum |terms|. The weight: one rounding of p and of p - decay, 2^-23 |p|, and the update
through a quotient, a root and the corrections, 2^-18 of it. Its bf16 copy is the rounding of the p that
came out, exactly. 8-bit moments: the
fp32 values before rounding are within 4 half steps of the terms' magnitudes of fp64's, e = 2^-22 sum
|terms| (which is large beside a value that came out of a cancellation), and the sum that places a
value below 2^-6 among its steps is rounded by at most 2^-21 of a step, less than one of the 65536 places of
the border. A code is the oracle's unless x - e and x + e, or the places beside the border, give another one;
it is then one of those."""
import numpy as np
import pytest
import torch

from oracle import lowbit

pytestmark = pytest.mark.gpu

HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


def api():
    from paper_2609_32415_gb300 import api as a
    return a


def d64(t):
    return t.detach().double().cpu().numpy()


def tensor(n, g, grad=torch.float32, offset=0, scale=1e-3):
    """One tensor's dict with fp32 moments; offset: elements by which every part lies behind an aligned address."""
    def part(dtype, s, make=torch.randn):
        return (make(n + offset, generator=g) * s).to(dtype).cuda()[offset:]
    return {"p": part(torch.float32, 0.02), "g": part(grad, scale), "m": part(torch.float32, 0.3 * scale),
            "v": part(torch.float32, scale * scale, torch.rand)}


def close(got, ref, tol):
    worst = float(np.max(np.abs(d64(got) - ref) / tol)) if ref.size else 0.0
    assert worst <= 1.0, worst


def check_step(before, after, lr, step, c=1.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01):
    g = d64(before["g"]) * c
    p0, m0, v0 = (d64(before[z]) for z in "pmv")
    p, m, v = lowbit.adamw(p0, g, m0, v0, lr, beta1, beta2, eps, weight_decay, step)
    close(after["m"], m, 2.0 ** -21 * (np.abs(m0) + np.abs(g)) + 1e-44)
    close(after["v"], v, 2.0 ** -21 * (v0 + g * g) + 1e-44)
    # a root's error near zero: v's own, through sqrt
    move = np.abs(lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps))
    spread = lr * 2.0 ** -21 * (np.abs(m0) + np.abs(g)) / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    close(after["p"], p, 2.0 ** -23 * np.abs(p0) + 2.0 ** -18 * move + spread + 1e-40)
    if "w" in after:
        assert torch.equal(after["w"], after["p"].bfloat16())


def cloned(t):
    return {k: v.clone() for k, v in t.items()}


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("step", [1, 2, 1000, 2000000])
@pytest.mark.parametrize("n", [1, 7, 8, 31, 33, 4096, 4097, 12289])
def test_32_bits(cuda_ok, grad, step, n):
    t = tensor(n, torch.Generator().manual_seed(n + step), grad)
    if n % 2:
        t["w"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    before = cloned(t)
    api().refadapt_adamw([t], 1e-3, step, **HYPER)
    check_step(before, t, 1e-3, step)


@pytest.mark.parametrize("offset", [1, 2, 4, 8])
def test_addresses_that_are_not_aligned(cuda_ok, offset):
    """The same bits as of aligned tensors."""
    a, g = api(), torch.Generator().manual_seed(offset)
    t = tensor(5000, g, torch.bfloat16, offset)
    u = {k: v.clone() for k, v in t.items()}
    a.refadapt_adamw([t], 1e-3, 3, **HYPER)
    a.refadapt_adamw([u], 1e-3, 3, **HYPER)
    assert all(torch.equal(t[k], u[k]) for k in t)


@pytest.mark.parametrize("hyper", [dict(beta1=0.0), dict(beta2=0.0), dict(weight_decay=0.0), dict(eps=1e-3),
                                   dict(beta1=0.99, beta2=0.95)])
def test_other_rates(cuda_ok, hyper):
    t = tensor(1000, torch.Generator().manual_seed(5))
    before = cloned(t)
    api().refadapt_adamw([t], 2e-2, 7, **{**HYPER, **hyper})
    check_step(before, t, 2e-2, 7, **{**HYPER, **hyper})


def test_many_tensors_in_one_call(cuda_ok):
    """More than one launch takes, empty ones among them; every tensor as alone."""
    a, g = api(), torch.Generator().manual_seed(6)
    sizes = [int(n) for n in torch.randint(0, 300, (700,), generator=g)]
    sizes[3], sizes[300], sizes[-1] = 0, 9001, 0
    ts = [tensor(n, g, torch.bfloat16 if i % 3 else torch.float32) for i, n in enumerate(sizes)]
    alone = [cloned(t) for t in ts]
    a.refadapt_adamw(ts, 1e-3, 4, **HYPER)
    for t, u in zip(ts, alone):
        a.refadapt_adamw([u], 1e-3, 4, **HYPER)
        assert all(torch.equal(t[k], u[k]) for k in t)
    a.refadapt_adamw([], 1e-3, 4)


def test_gradient_scale_and_skipped_steps(cuda_ok):
    a, g = api(), torch.Generator().manual_seed(8)
    t = tensor(3000, g)
    for c in (0.25, 0.0, float("nan"), float("inf")):
        before = cloned(t)
        a.refadapt_adamw([t], 1e-3, 9, grad_scale=torch.tensor([c], device="cuda"), **HYPER)
        if np.isfinite(c):
            check_step(before, t, 1e-3, 9, c)
        else:
            assert all(torch.equal(t[k], before[k]) for k in t)


# ------------------------------------------------------------------ 8 bits
def state8(x, floor=False):
    """(e4m3 tensor, e8m0 tensor) nearest to a flat fp64 array."""
    code, byte = lowbit.moment8(x, np.full(x.size, 32767.0), floor)
    return (torch.tensor(code.astype(np.uint8)).cuda().view(torch.float8_e4m3fn),
            torch.tensor(byte.astype(np.uint8)).cuda().view(torch.float8_e8m0fnu))


def small(t):
    """The dict with its moments in 8 bits."""
    u = {k: t[k].clone() for k in t}
    for z in "mv":
        u[z], u[z + "_scale"] = state8(d64(t[z]), z == "v")
    return u


def codes_of(t):
    return t.view(torch.uint8).cpu().numpy().astype(np.int64)


def moments_of(t):
    return {z: lowbit.values8(codes_of(t[z]), codes_of(t[z + "_scale"])) for z in "mv"}


def signed(code):
    """e4m3 codes in the order of their values."""
    return np.where(code & 128, -(code & 127), code & 127)


def check_step8(before, after, lr, step, seed, first, c=1.0):
    old = moments_of(before)
    full = {"p": before["p"], "g": before["g"], **{z: torch.tensor(old[z]) for z in "mv"}}
    g = d64(full["g"]) * c
    p, m, v = lowbit.adamw(d64(full["p"]), g, old["m"], old["v"], lr, 0.9, 0.999, 1e-8, 0.01, step)
    move = np.abs(lr * (m / (1 - 0.9 ** step)) / (np.sqrt(v / (1 - 0.999 ** step)) + 1e-8))
    spread = lr * 2.0 ** -21 * (np.abs(old["m"]) + np.abs(g)) / (1 - 0.9 ** step) / (np.sqrt(v / (1 - 0.999 ** step)) + 1e-8)
    close(after["p"], p, 2.0 ** -23 * np.abs(d64(full["p"])) + 2.0 ** -18 * move + spread + 1e-40)
    r = lowbit.random_bits(first, p.size, seed, step)
    for z, x, bits, floor in (("m", m, r & np.uint64(0xffff), False), ("v", v, r >> np.uint64(16), True)):
        byte, got = codes_of(after[z + "_scale"]), codes_of(after[z])
        assert np.array_equal(byte, lowbit.moment8_scales(x))
        e = 2.0 ** -22 * (np.abs(old["m"]) + np.abs(g) if z == "m" else old["v"] + g * g)
        e, bits = np.where(np.isfinite(e), e, 0.0), bits.astype(np.float64)
        near = [signed(lowbit.moment8_codes(y, byte, b, floor)) for y in (x - e, x + e) for b in (bits - 1, bits + 1)]
        low, high = np.min(near, 0), np.max(near, 0)  # x may lie on the other side of zero too
        assert np.all((low <= signed(got)) & (signed(got) <= high))
        assert np.sum(low != high) <= 1 + 0.01 * p.size  # of the oracle: nearly all codes are decided


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 8, 31, 32, 33, 100, 4096, 4129])
def test_8_bits(cuda_ok, grad, n):
    t = small(tensor(n, torch.Generator().manual_seed(n), grad))
    t["w"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    before = cloned(t)
    seed = (n << 40) + 12345
    api().refadapt_adamw([t], 1e-3, 12, seed=seed, **HYPER)
    check_step8(before, t, 1e-3, 12, seed, 0)
    assert torch.equal(t["w"], t["p"].bfloat16())


def test_8_bits_of_several_tensors(cuda_ok):
    """Random numbers go on from tensor to tensor, from a multiple of 32 on, and over launches."""
    a, g = api(), torch.Generator().manual_seed(31)
    ts = [small(tensor(n, g)) for n in [5, 0, 100] + [1] * 260 + [77]]
    before = [cloned(t) for t in ts]
    a.refadapt_adamw(ts, 1e-3, 2, seed=99, **HYPER)
    first = 0
    for t, b in zip(ts, before):
        n = t["p"].numel()
        if n:
            check_step8(b, t, 1e-3, 2, 99, first)
        first += -(-n // 32) * 32


@pytest.mark.parametrize("offset", [1, 4, 8])
def test_8_bits_not_aligned(cuda_ok, offset):
    a, g = api(), torch.Generator().manual_seed(offset)
    t = small(tensor(3000, g))
    u = {}
    for k, x in t.items():
        raw = torch.zeros(x.numel() + offset, dtype=torch.uint8 if x.element_size() == 1 else x.dtype, device="cuda")
        u[k] = raw[offset:].view(x.dtype) if x.element_size() == 1 else raw[offset:]
        u[k].view(raw.dtype).copy_(x.view(raw.dtype))
    a.refadapt_adamw([t], 1e-3, 3, **HYPER)
    a.refadapt_adamw([u], 1e-3, 3, **HYPER)
    for k in t:
        assert torch.equal(t[k].view(torch.uint8), u[k].contiguous().view(torch.uint8))


def test_8_bit_extremes(cuda_ok):
    """Zeros, the largest and smallest moments, a second moment that would round to zero, values that are not
    finite in one block."""
    n = 160
    t = {"p": torch.ones(n, device="cuda"), "g": torch.zeros(n, device="cuda")}
    m, v = np.zeros(n), np.zeros(n)
    m[32:64], v[32:64] = 1e-12, 1e-30                     # a tiny block
    m[64], v[64:96] = 1e4, 2.0 ** -30                     # one large value, and second moments far below
    v[64] = 1e8
    for z, x in (("m", m), ("v", v)):
        t[z], t[z + "_scale"] = state8(x, z == "v")
    t["g"][100] = float("inf")
    before = cloned(t)
    api().refadapt_adamw([t], 1e-3, 5, seed=1, **HYPER)
    after = moments_of(t)
    assert np.all(after["v"][64:96] > 0) and np.all(after["v"][32:64] > 0)
    assert np.isnan(after["m"][96:128]).all() and np.isnan(after["v"][96:128]).all()
    rest = np.r_[0:96, 128:160]
    assert np.isfinite(after["m"][rest]).all() and np.isfinite(d64(t["p"])[rest]).all()
    assert np.all(after["m"][:32] == 0) and np.all(after["v"][:32] == 0)
    part = {k: x[:3] if "scale" in k else x[:96] for k, x in before.items()}
    check_step8(part, {k: x[:3] if "scale" in k else x[:96] for k, x in t.items()}, 1e-3, 5, 1, 0)


def test_8_bit_moments_keep_their_mean(cuda_ok):
    """Steps without a gradient: v decays as beta2^t although a step is far below a step of its format. Each step
    rounds with a variance of at most p (1 - p) s^2, p the part of a step s that it decays by (0.001 v / s), so v's
    variance after t steps is at most t 0.001 v s <= t 1e-3 v^2 / 8; over n independent values the mean's deviation
    is below sqrt(t 1e-3 / 8 / n): 5 deviations are allowed."""
    a, n, steps = api(), 1 << 16, 400
    t = {"p": torch.zeros(n, device="cuda"), "g": torch.zeros(n, device="cuda")}
    x = np.random.default_rng(0).uniform(1.0, 1.9, n)
    for z in "mv":
        t[z], t[z + "_scale"] = state8(x, z == "v")
    v0 = moments_of(t)["v"]
    for k in range(steps):
        a.refadapt_adamw([t], 0.0, k + 1, seed=7, **HYPER)
    ratio = moments_of(t)["v"].mean() / (v0.mean() * 0.999 ** steps)
    assert abs(ratio - 1) < 5 * np.sqrt(steps * 1e-3 / 8 / n) + 1e-4, ratio


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("sizes", [[], [0], [1], [4095, 1, 4097], [100000, 3, 0, 77] + [5] * 600])
@pytest.mark.parametrize("most", [0.5, 1e9, float("inf")])
def test_norm(cuda_ok, sizes, most):
    a, g = api(), torch.Generator().manual_seed(len(sizes))
    grads = [torch.randn(n + i % 2, generator=g).to(torch.bfloat16 if i % 3 else torch.float32).cuda()[i % 2:]
             for i, n in enumerate(sizes)]
    out, ws = torch.full((2,), 7.0, device="cuda"), a.grad_norm_workspace()
    for _ in range(2):  # the workspace is ready again
        a.refadapt_grad_norm(grads, most, out, ws)
        want = np.sqrt(sum(float((d64(t) ** 2).sum()) for t in grads))
        # 32 fp32 sums in a row, the rest in fp64: 33 half steps of the squares, half of that in the root: 2^-19.9
        assert abs(float(out[0]) - want) <= 2.0 ** -19 * want
        clip = most / want if want > most else 1.0
        assert abs(float(out[1]) - clip) <= 2.0 ** -19 * clip


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 1e20])
def test_norm_that_is_not_finite_skips_the_step(cuda_ok, bad):
    a, g = api(), torch.Generator().manual_seed(3)
    t = tensor(9000, g)
    t["g"][8999] = bad
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    before = cloned(t)
    a.refadapt_grad_norm([t["g"]], 1.0, out, ws)
    a.refadapt_adamw([t], 1e-3, 1, grad_scale=out[1:], **HYPER)
    assert np.isnan(float(out[1])) and all(torch.equal(t[k], before[k]) for k in "pmv")


def test_norm_is_the_same_every_time(cuda_ok):
    a, g = api(), torch.Generator().manual_seed(4)
    grads = [torch.randn(n, generator=g).cuda() for n in (1000003, 77, 300000)]
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    seen = set()
    for _ in range(20):
        a.refadapt_grad_norm(grads, 1.0, out, ws)
        seen.add((float(out[0]), float(out[1])))
    assert len(seen) == 1


# ------------------------------------------------------------------ a captured step
@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_go_on(cuda_ok, bits):
    """Norm and step in a graph that reads its rate and number from the device: replays are the eager steps."""
    a, g = api(), torch.Generator().manual_seed(13)
    ts = [tensor(n, g) for n in (5000, 33)]
    ts = [small(t) if bits == 8 else t for t in ts]
    eager = [cloned(t) for t in ts]
    lr, step = torch.tensor([1e-3], device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()

    def one(tensors, lr, step):
        a.refadapt_grad_norm([t["g"] for t in tensors], 0.05, out, ws)
        a.refadapt_adamw(tensors, lr, step, grad_scale=out[1:], seed=21, **HYPER)

    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        one(ts, lr, step)
        step.add_(1)
    for k in range(3):
        graph.replay()
        lr.mul_(0.5)
    torch.cuda.synchronize()
    for k in range(3):
        one(eager, 1e-3 * 0.5 ** k, k + 1)
    for t, u in zip(ts, eager):
        assert all(torch.equal(t[k].view(torch.uint8), u[k].view(torch.uint8)) for k in t)
    assert int(step) == 4
