"""A wait that runs out in refadapt_gemm: one output tile with a K so long that the
epilogue gives up (after two turns of 10 us at least, however short the budget) while the
loads and MMAs go on. The CTA lets them land, the error word is set, and the next call
gives what the first gave."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile_mode", [1, 2])
def test_a_wait_that_runs_out(cuda_ok, tile_mode):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RA_EPI_STORE, RA_ETIMEOUT, RefAdaptError
    g = torch.Generator(device="cuda").manual_seed(tile_mode)
    n, K, N = 256, 65536, 256
    a = torch.randn((1, n, K), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((N, K), generator=g, device="cuda") / 256).to(torch.bfloat16)
    out = torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        api.refadapt_gemm([{"a": a, "w": w, "out": out}], N, K, RA_EPI_STORE, err_word=err, tile_mode=tile_mode)

    call()
    api.refadapt_check_error(err)
    want = out.clone()
    api.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(3):
            out.fill_(float("nan"))
            call()
            with pytest.raises(RefAdaptError) as e:
                api.refadapt_check_error(err)
            assert e.value.status == RA_ETIMEOUT
    finally:
        api.refadapt_set_wait_budget_ns(500_000_000)
    call()
    api.refadapt_check_error(err)
    assert torch.equal(out, want)
