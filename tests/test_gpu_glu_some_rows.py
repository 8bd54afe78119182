"""The gated feed-forward's forward pass at the row counts and widths around its three forms:
rows that stream the weights (up to 16 and small weights), rows as the product's columns (up to
128), tiles (more); and the backward pass around its two forms. Tolerances as in test_gpu_glu.py."""
import numpy as np
import pytest
import torch

from _helpers import f64
from test_gpu_glu import call, check_forward, check_grads, grads, seg

pytestmark = pytest.mark.gpu


def run(segs, F, C, act, **kw):
    from paper_2609_32415_gb300 import api
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.refadapt_glu(segs, F, C, act, err_word=err, **kw)
    api.refadapt_check_error(err)
    return api.refadapt_last_launch()


@pytest.mark.parametrize("rows,C,F,form", [
    (9, 64, 64, "few"), (16, 1000, 2736, "few"), (16, 2048, 3200, "some"), (8, 4096, 4104, "some"),
    (17, 64, 64, "some"), (17, 72, 72, "some"), (24, 136, 1224, "some"), (63, 520, 2440, "some"), (96, 2056, 1216, "some"),
    (112, 1536, 9736, "some"), (113, 200, 20000, "some"), (128, 64, 2728, "some"), (129, 64, 264, "CTA pairs")])
@pytest.mark.parametrize("save", [False, True])
def test_forms(cuda_ok, rows, C, F, form, save):
    g = torch.Generator().manual_seed(rows + C + F)
    s = seg(1, rows, C, F, g, save)
    assert run([s], F, C, rows % 2).startswith(form)
    check_forward(s, rows % 2)


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("B,rows", [(2, 9), (3, 31), (5, 17), (8, 16), (16, 3)])
def test_samples(cuda_ok, B, rows, strided):
    """Samples that follow one another share columns; others have a multiple of eight each."""
    g = torch.Generator().manual_seed(B + rows)
    C, F = 264, 1368
    s = seg(B, rows, C, F, g, True, strided)
    assert run([s], F, C, 0).startswith("some")
    check_forward(s, 0)


def test_segments_and_modes(cuda_ok):
    g = torch.Generator().manual_seed(5)
    B, C, F = 2, 392, 1000
    segs = [seg(B, 7, C, F, g, False, True), seg(B, 30, C, F, g, True), seg(B, 64, C, F, g, False)]
    segs[1]["gated"] = True
    segs[1]["out"].fill_(float("nan")), segs[1]["pre_up"].fill_(float("nan"))
    mode = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    assert run(segs, F, C, 1, mode=mode).startswith("some")
    for i, s in enumerate(segs):
        check_forward(s, 1, skip=(1,) if i == 1 else ())


@pytest.mark.parametrize("rows", [17, 40, 127])
def test_nan_and_infinity_stay_in_their_row(cuda_ok, rows):
    g = torch.Generator().manual_seed(rows)
    C, F = 200, 328
    s = seg(1, rows, C, F, g, False)
    s["x"][0, 3, 5], s["x"][0, rows - 1, 199] = float("nan"), float("inf")
    run([s], F, C, 0)
    out = f64(s["out"])[0]
    bad = [3, rows - 1]
    assert np.isnan(out[3]).all() and not np.isfinite(out[rows - 1]).all()
    rest = [r for r in range(rows) if r not in bad]
    part = {"x": s["x"][:, rest], "w_gate": s["w_gate"], "w_up": s["w_up"], "out": s["out"][:, rest]}
    check_forward(part, 0)


def test_the_same_bits_on_every_call(cuda_ok):
    g = torch.Generator().manual_seed(1)
    C, F = 2048, 5504
    s = seg(1, 50, C, F, g, True)
    run([s], F, C, 0)
    first = {k: s[k].clone() for k in ("out", "pre_gate", "pre_up")}
    for _ in range(20):
        run([s], F, C, 0)
        for k, v in first.items():
            assert torch.equal(s[k], v), k


EVERY = ("dx", "dw_gate", "dw_up", "dw_down")


@pytest.mark.parametrize("B,n,C,F,O,strided", [
    (1, 3, 2048, 72, 64, False), (1, 16, 520, 2736, 264, True), (2, 8, 72, 1000, 2056, False), (1, 17, 520, 1000, 1032, False),
    (4, 16, 264, 648, 136, True), (1, 64, 1024, 1368, 200, False), (1, 65, 1024, 1368, 200, False)])
@pytest.mark.parametrize("want", [EVERY, ("dx",), ("dx", "dw_up")])
def test_backward(cuda_ok, B, n, C, F, O, strided, want):
    run_backward(B, n, C, F, O, strided, want, n % 2)


@pytest.mark.parametrize("B,n,C,F,O,strided", [
    (1, 129, 1000, 2000, 1096, False), (1, 256, 264, 4104, 520, True), (3, 85, 136, 712, 264, True),
    (1, 257, 264, 712, 128, False), (200, 1, 128, 200, 72, True)])
def test_input_gradient_alone(cuda_ok, B, n, C, F, O, strided):
    run_backward(B, n, C, F, O, strided, ("dx",), n % 2)


def run_backward(B, n, C, F, O, strided, want, act):
    from paper_2609_32415_gb300 import api
    g = torch.Generator().manual_seed(n + C + F + O)
    s = grads(B, n, C, F, O, g, act, strided)
    ws = torch.full((api.refadapt_glu_backward_workspace_size(B, n, C, F, O) // 2,), float("nan"), dtype=torch.bfloat16,
                    device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    drop = [k for k in EVERY if k not in want]
    call(s, act, ws, err, drop)
    api.refadapt_check_error(err)
    check_grads(s, act, drop)
    first = {k: s[k].clone() for k in want}
    for _ in range(3):
        call(s, act, ws, err, drop)
        for k, v in first.items():
            assert torch.equal(s[k], v), k
