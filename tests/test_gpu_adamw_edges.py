"""The optimiser's step and the norm over whole chunks of elements (the loads of several are on their way at once there),
and at the ends of fp32's range. Bounds as in test_gpu_adamw."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import HYPER, api, check_step, check_step8, cloned, d64, small, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [8192, 8193, 3 * 8192 + 77, 65536])
def test_whole_chunks_in_8_bits(cuda_ok, grad, n):
    t = small(tensor(n, torch.Generator().manual_seed(n), grad))
    t["w"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    before = cloned(t)
    api().refadapt_adamw([t], 1e-3, 12, seed=(5 << 33) + n, **HYPER)
    check_step8(before, t, 1e-3, 12, (5 << 33) + n, 0)
    assert torch.equal(t["w"], t["p"].bfloat16())


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [8192, 3 * 8192 + 77])
def test_whole_chunks_behind_another_tensor(cuda_ok, grad, n):
    """Chunks of the second tensor of a call, whose random numbers go on from the first."""
    g = torch.Generator().manual_seed(n)
    ts = [small(tensor(100, g)), small(tensor(n, g, grad))]
    before = [cloned(t) for t in ts]
    api().refadapt_adamw(ts, 1e-3, 3, seed=17, **HYPER)
    for t, b, first in zip(ts, before, (0, 128)):
        check_step8(b, t, 1e-3, 3, 17, first)


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[8192], [5 * 8192 + 1234], [8192, 3, 2 * 8192 + 9, 8192], [152 * 8 * 8192 + 3 * 8192 + 5]])
def test_norm_of_whole_chunks(cuda_ok, grad, sizes):
    """Each type's whole chunks, remainders, and more chunks than CTAs."""
    a, g = api(), torch.Generator().manual_seed(len(sizes))
    grads = [torch.randn(n, generator=g).to(grad).cuda() for n in sizes]
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    for _ in range(2):
        a.refadapt_grad_norm(grads, 0.5, out, ws)
        want = np.sqrt(sum(float((d64(t) ** 2).sum()) for t in grads))
        assert abs(float(out[0]) - want) <= 2.0 ** -19 * want
        assert abs(float(out[1]) - 0.5 / want) <= 2.0 ** -19 * 0.5 / want


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 8192 + 64])
@pytest.mark.parametrize("top", [1e15, 1.5e17, 1e18, 1.8e19])
def test_large_gradients_move_the_weights(cuda_ok, bits, grad, n, top):
    """Squares up to the end of fp32: the step is lr times a number near one for them, and what it was for the
    ordinary gradients beside them."""
    g = torch.Generator().manual_seed(7)
    t = tensor(n, g, grad)
    large = torch.arange(0, n, 3, device="cuda")
    t["g"][large] = (torch.sign(t["g"][large].float()) * top).to(grad)
    if bits == 8:
        t = small(t)
    before = cloned(t)
    api().refadapt_adamw([t], 1e-3, 12, seed=3, **HYPER)
    if bits == 8:
        check_step8(before, t, 1e-3, 12, 3, 0)
    else:
        check_step(before, t, 1e-3, 12)
    assert bool(((t["p"] - before["p"])[large].abs() > 1e-4).all())


def test_large_moments_move_the_weights(cuda_ok):
    """Second moments from 2^100 to the end of fp32, without a gradient."""
    n = 64
    v = (2.0 ** torch.linspace(90, 127.9, n, dtype=torch.float64)).float().cuda()
    t = {"p": torch.ones(n, device="cuda"), "g": torch.zeros(n, device="cuda"), "m": v.sqrt(), "v": v}
    before = cloned(t)
    api().refadapt_adamw([t], 1e-2, 2, **HYPER)
    check_step(before, t, 1e-2, 2)
    assert bool(((t["p"] - before["p"]).abs() > 1e-5).all())


@pytest.mark.parametrize("eps", [1.2e-38, 1e-30])
def test_smallest_eps_and_tiny_gradients(cuda_ok, eps):
    """Elements whose moments are zero stay where they are but for the decay; the roots of the smallest second moments
    are not lost beside such an eps."""
    n = 256
    t = {"p": torch.ones(n, device="cuda"), "g": torch.zeros(n, device="cuda"), "m": torch.zeros(n, device="cuda"),
         "v": torch.zeros(n, device="cuda")}
    t["v"][128:] = (2.0 ** torch.linspace(-126, -100, 128, dtype=torch.float64)).float().cuda()
    t["m"][128:] = t["v"][128:].sqrt() * 0.5
    before = cloned(t)
    api().refadapt_adamw([t], 1e-3, 4, **{**HYPER, "eps": eps})
    check_step(before, t, 1e-3, 4, eps=eps)
    assert bool((t["p"][:128] == t["p"][0]).all()) and abs(float(t["p"][0]) - (1 - 1e-5)) < 1e-6


@pytest.mark.parametrize("tensors", [0, 3, 600])
def test_workspace_counts_finite_norms(cuda_ok, tensors):
    """Once a call, whatever its launches; a step reads its number there."""
    a, g = api(), torch.Generator().manual_seed(2)
    grads = [torch.randn(50, generator=g).cuda() for _ in range(tensors)]
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    count = ws[4:8].view(torch.int32)
    t = tensor(100, g)
    u = cloned(t)
    for k, bad in enumerate([False, True, False, True, True, False]):
        if tensors:
            grads[-1][7] = float("inf") if bad else 1.0
        a.refadapt_grad_norm(grads, 1.0, out, ws)
        a.refadapt_adamw([t], 1e-3, count, grad_scale=out[1:], **HYPER)
    taken = 3 if tensors else 6
    assert int(count) == taken
    if tensors:
        grads[-1][7] = 1.0
    fresh = a.grad_norm_workspace()
    for k in range(taken):
        a.refadapt_grad_norm(grads, 1.0, out, fresh)
        a.refadapt_adamw([u], 1e-3, k + 1, grad_scale=out[1:], **HYPER)
    assert all(torch.equal(t[z], u[z]) for z in t)
