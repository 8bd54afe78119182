"""Offsets past 32 bits in the 4-bit calls and in the optimiser's: the last rows or elements are what they
are in a small call, which other tests check. Up to 60 GB on the device."""
import pytest
import torch

from test_gpu_adamw import HYPER, check_step, check_step8, cloned, small, tensor

pytestmark = pytest.mark.gpu
E4M3, E8M0 = 0, 1


def api():
    from paper_2609_32415_gb300 import api as a
    return a


def bytes_(*shape):
    return torch.empty(shape, dtype=torch.uint8, device="cuda")


@pytest.fixture
def room(cuda_ok):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of free memory")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt", [E4M3, E8M0])
def test_quantisation(room, fmt):
    a, n, C, times = api(), 512, 8192, 1025  # 4.3e9 values
    base = torch.randn((1, n, C), device="cuda", generator=torch.Generator("cuda").manual_seed(fmt)).bfloat16()
    x = base.repeat(1, times, 1)
    rows = n * times

    def run(x, rows):
        codes, scales = a.quant4_buffers(1, rows, C, fmt)
        seg = {"x": x, "codes": codes, "scales": scales, "codes_t": bytes_(C, rows // 2),
               "scales_t": bytes_(a.refadapt_quant4_scales_size(C, rows, fmt))}
        a.refadapt_quant4([seg], C, fmt)
        alone = torch.full_like(codes, 7)  # along the features only: another kernel
        a.refadapt_quant4([{"x": x, "codes": alone, "scales": torch.empty_like(scales)}], C, fmt)
        return seg, alone

    want, _ = run(base, n)
    got, alone = run(x, rows)
    for i in (0, times // 2, times - 1):
        for codes in (got["codes"], alone):
            assert torch.equal(codes[:, i * n:(i + 1) * n], want["codes"])
        assert torch.equal(got["scales"][:, i * n // 128:(i + 1) * n // 128], want["scales"])
        assert torch.equal(got["codes_t"][:, i * n // 2:(i + 1) * n // 2], want["codes_t"])


@pytest.mark.parametrize("tile_mode", [1, 2])
def test_product(room, tile_mode):
    a, few, N, K, fmt = api(), 512, 32768, 64, E8M0
    rows = few * 274  # 4.6e9 results
    g = torch.Generator("cuda").manual_seed(3)
    x, w = (torch.randn(s, device="cuda", generator=g).bfloat16() for s in ((1, few, K), (1, N, K)))
    codes = [a.quant4_buffers(1, n, K, fmt) for n in (few, N, rows)]
    for x_, (c, s) in zip((x, w, x.repeat(1, rows // few, 1)), codes):
        a.refadapt_quant4([{"x": x_, "codes": c, "scales": s}], K, fmt)
    outs = []
    for (c, s), n in ((codes[0], few), (codes[2], rows)):
        outs.append(torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda"))
        a.refadapt_gemm4([{"a": c, "a_scales": s, "w": codes[1][0][0], "w_scales": codes[1][1][0], "out": outs[-1]}], N, K, 0, fmt,
                         tile_mode=tile_mode)
    for i in (0, 137, 273):
        assert torch.equal(outs[1][:, i * few:(i + 1) * few], outs[0])


def big(n, tail, bits):
    """A tensor of n zeros but for its last elements, those of `tail`; and what of it they are."""
    a, k = api(), tail["p"].numel()
    t = {"p": torch.zeros(n, device="cuda"), "g": torch.zeros(n, dtype=tail["g"].dtype, device="cuda")}
    t.update(a.adamw_moments(t["p"], bits))
    part = {z: v[-(-(-k // 32) if z.endswith("scale") else k):] for z, v in t.items()}
    for z, v in part.items():
        v.view(torch.uint8).copy_(tail[z].view(torch.uint8))
    return t, part


def test_32_bit_moments_and_norm(room):
    a, k = api(), 4096 + 77
    tail = tensor(k, torch.Generator().manual_seed(8), torch.bfloat16)
    t, part = big((1 << 31) + 8 * 1001 + k, tail, 32)
    a.refadapt_adamw([t], 1e-3, 5, **HYPER)
    check_step(tail, part, 1e-3, 5)
    assert int(torch.count_nonzero(t["p"][:-k])) == 0
    out, ws = torch.zeros(2, device="cuda"), a.grad_norm_workspace()
    a.refadapt_grad_norm([t["g"]], 1.0, out, ws)
    want = float(tail["g"].double().square().sum().sqrt())
    assert abs(float(out[0]) - want) <= 2.0 ** -19 * want


def test_8_bit_moments(room):
    a, k = api(), 4096 + 77
    n = (1 << 32) + 32 * 1001 + k
    tail = small(tensor(k, torch.Generator().manual_seed(9), torch.bfloat16))
    t, part = big(n, tail, 8)
    before = cloned(part)
    a.refadapt_adamw([t], 1e-3, 5, seed=77, **HYPER)
    check_step8(before, part, 1e-3, 5, 77, n - k)
