"""refadapt_q_delta under a wait budget that no wait can be sure to meet: D is right or NaN
(a consumer gave up), the loads in flight have landed when the call ends, and the next call
gives what the first gave."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,n,d", [(1, 24, 4096, 128), (2, 8, 500, 64)])
@pytest.mark.parametrize("tokens", [False, True])
def test_a_budget_that_no_wait_is_sure_to_meet(cuda_ok, B, H, n, d, tokens):
    from paper_2609_32415_gb300 import api
    g = torch.Generator(device="cuda").manual_seed(n)
    shape = (B, n, H, d) if tokens else (B, H, n, d)
    cur, prev = (torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    if tokens:
        cur, prev = cur.transpose(1, 2), prev.transpose(1, 2)
    D, ws = torch.empty((B, H), device="cuda"), api.q_delta_workspace(B, H)
    api.refadapt_q_delta(cur, prev, D, ws)
    want = D.clone()
    api.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(10):
            D.zero_()
            api.refadapt_q_delta(cur, prev, D, ws)
            assert bool(((D == want) | torch.isnan(D)).all())
    finally:
        api.refadapt_set_wait_budget_ns(500_000_000)
    api.refadapt_q_delta(cur, prev, D, ws)
    assert torch.equal(D, want)
