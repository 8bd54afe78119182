"""The backward pass of the residual norm over long runs of rows, and around its shift.

A CTA's rows pass through slots between warps that reduce rows and groups of warps that take
columns; the widths here give one, two, three, five and ten such groups, the row counts many
turns of every slot, and the kinds of norms rows that are reduced quickly and slowly. Sums
over a row are taken around the mean of its first eight values.
"""
import pytest
import torch

from test_gpu_block_layers import GRADS, backward_case, bf, check_backward, norm_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("post,pre", [(0, 0), (0, 1), (1, 2), (1, 1)])
@pytest.mark.parametrize("C,B,n", [(200, 1, 9001), (504, 2, 4500), (640, 1, 9000), (768, 1, 9000), (1160, 1, 6100),
                                   (2560, 1, 4700)])
def test_long_runs(cuda_ok, C, B, n, post, pre):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(C + n + 10 * post + pre)
    s = norm_case(B, n, C, g, True)
    s["dx"], s["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case(s, n, C, B)
    ws = api.residual_norm_backward_workspace(B, n, C)
    api.refadapt_residual_norm_backward(s, C, post, pre, ws)
    first = {k: s[k].clone() for k in GRADS if k in s}
    # dh and dy are per row: a sample of the rows is enough for the 64-bit form
    take = torch.arange(0, n, 7)
    part = {k: v[:, take] if torch.is_tensor(v) and v.dim() == 3 else v for k, v in s.items()}
    check_backward({k: v for k, v in part.items() if k not in GRADS or k in ("dh", "dy")}, post, pre, 1e-6, 1.0)
    for _ in range(20):  # whichever warps are ahead: the same bits
        api.refadapt_residual_norm_backward(s, C, post, pre, ws)
        for k, v in first.items():
            assert torch.equal(s[k], v), k


@pytest.mark.parametrize("post,pre", [(1, 1), (2, 1), (1, 2)])
@pytest.mark.parametrize("C", [1160, 5120])
@pytest.mark.parametrize("offset", [64.0, -3000.0])
def test_first_columns_far_from_the_rest(cuda_ok, post, pre, C, offset):
    """Around those eight values' mean a row's sum of squares is at most C / 8 + 1 times
    that around its own mean, so its variance is good to (C / 8 + 1) times the sum's own
    rounding (2^-24 a term at a chain of at most 100): 4e-3 at worst, and 2^-12 in practice
    (roundings that do not all add up), under a bf16 result's 2^-9."""
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(C)
    B, n = 1, 40
    s = norm_case(B, n, C, g, True)
    for k in ("h", "y"):
        s[k][:, :, :8] += offset
    s["dx"], s["dh_out"] = bf((B, n, C), g), bf((B, n, C), g)
    s = backward_case(s, n, C, B, ("dgate", "dscale", "dshift", "dpost_w", "dpre_w"))
    api.refadapt_residual_norm_backward(s, C, post, pre, api.residual_norm_backward_workspace(B, n, C))
    check_backward(s, post, pre, 1e-6, 1.0)
