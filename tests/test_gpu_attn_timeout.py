"""The joint attention under a wait budget that no wait can be sure to meet: a call either
ends right or says in its error word that it gave up; what it had in flight has landed when
it ends, and the next call gives what the first gave. Shapes of one launch form each."""
import pytest
import torch

from _helpers import ROLES, empty_outputs, make_segments

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,n", [(24, dict(text=256, ref=4096, tgt=2048)), (3, dict(text=33, ref=300, tgt=127)),
                                 (8, dict(text=77, ref=1000, tgt=500))])
def test_a_budget_that_no_wait_is_sure_to_meet(cuda_ok, H, n):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RA_ETIMEOUT, RefAdaptError
    B, d = 1, 128
    segs = make_segments(B, H, d, n, gen=torch.Generator().manual_seed(H))
    mp = torch.zeros((B, H, api.refadapt_mass_partial_len(n["text"], n["tgt"])), device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        out = empty_outputs(B, H, d, n)
        api.refadapt_joint_attn(*([segs[r][z] for r in ROLES] for z in range(3)), [out[r] for r in ROLES], mp,
                                err_word=err)
        return [out[r] for r in ROLES]

    want = call()
    api.refadapt_check_error(err)
    api.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(5):
            got = call()
            try:
                api.refadapt_check_error(err)
            except RefAdaptError as e:
                assert e.status == RA_ETIMEOUT
            else:
                assert all(torch.equal(a, b) for a, b in zip(got, want))
    finally:
        api.refadapt_set_wait_budget_ns(500_000_000)
    got = call()
    api.refadapt_check_error(err)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
