"""A wait that runs out in a kernel of the gated feed-forward: the call ends, its error
word says so, the context stays usable and the next call gives what the first gave.

Each case has one product whose K is so long that the epilogue's wait for its
accumulator (two turns of 10 us at least, however short the budget) cannot be met, while
the loads and MMAs go on: a CTA that gives up lets them land before it exits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def bf(*shape, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def forward(rows, form):
    from paper_2609_32415_gb300 import api
    C, F = 65536, 64
    x, w, out = bf(1, rows, C), [bf(F, C, scale=C ** -0.5), bf(F, C, scale=-C ** -0.5)], bf(1, rows, F)

    def call(err):
        api.refadapt_glu([{"x": x, "w_gate": w[0], "w_up": w[1], "out": out}], F, C, 0, err_word=err)
        assert api.refadapt_last_launch().startswith(form), api.refadapt_last_launch()
        return [out]

    return call


def backward(rows, C, F, O, want):
    from paper_2609_32415_gb300 import api
    dy, x, g, w, u = bf(1, rows, O), bf(1, rows, C), bf(1, rows, F), bf(1, rows, F, scale=0.5), bf(1, rows, F)
    weights = [bf(F, C, scale=C ** -0.5), bf(F, C, scale=-C ** -0.5), bf(O, F, scale=F ** -0.5)]
    ws = api.glu_backward_workspace(1, rows, C, F, O)
    out = {"dx": bf(1, rows, C), "dw_gate": bf(F, C), "dw_up": bf(F, C), "dw_down": bf(O, F)}
    out = {k: v for k, v in out.items() if k in want}

    def call(err):
        api.refadapt_glu_backward(dy, x, *weights, g, w, u, 0, ws, err_word=err, **out)
        return list(out.values())

    return call


CASES = {
    "CTA pairs": lambda: forward(256, "CTA pairs"),
    "some rows": lambda: forward(100, "some rows"),
    "dg and dw by tiles": lambda: backward(300, 64, 64, 1 << 18, ("dx", "dw_gate")),
    "dg and dw by clusters": lambda: backward(16, 64, 64, 1 << 18, ("dx",)),
    "dx by clusters": lambda: backward(16, 64, 1 << 18, 64, ("dx",)),
    "weights' gradients": lambda: backward(1000000, 64, 64, 64, ("dw_gate", "dw_up", "dw_down")),
}


@pytest.mark.parametrize("name", CASES)
def test_a_wait_that_runs_out(cuda_ok, name):
    from paper_2609_32415_gb300 import api
    from paper_2609_32415_gb300._lib import RA_ETIMEOUT, RefAdaptError
    call = CASES[name]()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = [t.clone() for t in call(err)]
    api.refadapt_check_error(err)
    api.refadapt_set_wait_budget_ns(1)
    try:
        for _ in range(3):
            for t in call(err):
                t.fill_(float("nan"))
            with pytest.raises(RefAdaptError) as e:
                api.refadapt_check_error(err)
            assert e.value.status == RA_ETIMEOUT
    finally:
        api.refadapt_set_wait_budget_ns(500_000_000)
    for a, b in zip(want, call(err)):
        assert torch.equal(a, b)
    api.refadapt_check_error(err)
