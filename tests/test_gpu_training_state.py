"""training.AdamW and training.linear4 as torch has them: gradients, graphs of older weights, steps that count."""
import pytest
import torch

from test_gpu_linear4 import E4M3, E8M0, bf

pytestmark = pytest.mark.gpu


def training():
    from paper_2609_32415_gb300 import training as t
    return t


@pytest.mark.parametrize("bits", [32, 8])
def test_a_graph_of_older_weights_raises(cuda_ok, bits):
    """A step writes parameters: a backward pass that would read one that it saved before raises, as after a step of
    torch's optimisers; parameters that a step left alone stay good."""
    t, g = training(), torch.Generator().manual_seed(1)
    w, v = torch.nn.Parameter(bf((64, 128), g, 0.1)), torch.nn.Parameter(torch.randn(50, generator=g).cuda())
    still = torch.nn.Parameter(bf((64, 128), g, 0.1))
    x = bf((1, 40, 128), g).requires_grad_(True)
    opt = t.AdamW([w, v, still], 1e-2, bits=bits)
    y, z, kept = t.linear4(x, w), (v * v).sum(), t.linear4(x, still)
    w.grad, v.grad = torch.ones_like(w), torch.ones_like(v)
    opt.step()
    for stale in (y.float().sum(), z):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            stale.backward()
    kept.float().sum().backward()
    assert still.grad is not None
    t.linear4(x, w).float().sum().backward()  # a graph of the new weights


@pytest.mark.parametrize("fmt, exps", [(E8M0, (0, 0)), (E4M3, (1, -5))])
def test_linear4_of_a_weight_in_a_wider_buffer(cuda_ok, fmt, exps):
    """Rows with a stride of their own, forward and backward: what the same weight gives on its own."""
    t, g = training(), torch.Generator().manual_seed(2)
    wide, x, up = bf((64, 256), g, 0.1), bf((2, 40, 128), g), bf((2, 40, 64), g)
    got = []
    for w in (wide[:, 64:192], wide[:, 64:192].contiguous()):
        w, xr = w.detach().requires_grad_(True), x.clone().requires_grad_(True)
        y = t.linear4(xr, w, fmt, *exps)
        got.append((y.detach(), *torch.autograd.grad(y, (xr, w), up)))
    for a, b in zip(*got):
        assert a.shape == b.shape and torch.equal(a, b)


def test_linear4_of_a_weight_in_a_wider_buffer_without_its_own_gradient(cuda_ok):
    t, g = training(), torch.Generator().manual_seed(3)
    wide, x, up = bf((64, 256), g, 0.1), bf((1, 40, 128), g), bf((1, 40, 64), g)
    xr = x.clone().requires_grad_(True)
    (dx,) = torch.autograd.grad(t.linear4(xr, wide[:, :128]), xr, up)
    xs = x.clone().requires_grad_(True)
    (want,) = torch.autograd.grad(t.linear4(xs, wide[:, :128].contiguous()), xs, up)
    assert torch.equal(dx, want)


def test_linear4_takes_the_weights_own_exponent(cuda_ok):
    """w_exponent None: the one that api.weight4 takes from the weight's largest magnitude."""
    from paper_2609_32415_gb300 import api
    t, g = training(), torch.Generator().manual_seed(4)
    x, w = bf((1, 40, 128), g), bf((64, 128), g, 0.02)
    exponent = api.weight4(w, E4M3).exponent
    assert exponent < 0
    assert torch.equal(t.linear4(x, w, E4M3, 0, None), t.linear4(x, w, E4M3, 0, exponent))


@pytest.mark.parametrize("capturable", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad_at", [0, 2])
def test_skipped_steps_do_not_count(cuda_ok, capturable, bits, bad_at):
    """A step whose gradients are not finite changes nothing: the steps behind it are those of a run without it."""
    t, g = training(), torch.Generator().manual_seed(5)
    start = [torch.randn(300, generator=g).cuda(), bf((20, 10), g)]
    grads = [[torch.randn(p.shape, generator=g).to(p.dtype).cuda() for p in start] for _ in range(4)]
    runs = []
    for skip in (False, True):
        params = [torch.nn.Parameter(p.clone()) for p in start]
        opt = t.AdamW(params, 1e-2, bits=bits, max_norm=1.0, seed=9, capturable=capturable)
        for k, step in enumerate(grads):
            if skip and k == bad_at:
                params[0].grad, params[1].grad = step[0].clone(), step[1].clone()
                params[0].grad[7] = float("nan")
                was = [p.detach().clone() for p in params]
                opt.step()
                assert all(torch.equal(p.detach(), q) for p, q in zip(params, was))
            for p, v in zip(params, step):
                p.grad = v.clone()
            opt.step()
        assert int(opt.count) == len(grads)
        runs.append((params, opt.state_dict()))
    for p, q in zip(runs[0][0], runs[1][0]):
        assert torch.equal(p.detach(), q.detach())
    assert int(runs[0][1]["count"]) == int(runs[1][1]["count"])


def test_a_captured_step_that_is_skipped_does_not_count(cuda_ok):
    t, g = training(), torch.Generator().manual_seed(6)
    start, grad = torch.randn(100, generator=g).cuda(), torch.randn(100, generator=g).cuda()
    p, q = (torch.nn.Parameter(start.clone()) for _ in range(2))
    one, two = (t.AdamW([z], 1e-2, max_norm=1.0, capturable=True) for z in (p, q))
    p.grad, q.grad = grad.clone(), grad.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        one.step()
    for bad in (True, False, True, False):
        p.grad.copy_(grad)
        if bad:
            p.grad[3] = float("inf")
        graph.replay()
    torch.cuda.synchronize()
    two.step()
    two.step()
    assert int(one.count) == 2 and torch.equal(p.detach(), q.detach())


@pytest.mark.parametrize("capturable", [False, True])
def test_refused_steps_do_not_count(cuda_ok, capturable):
    """Parameters that share memory: the call is refused, and count and weights stay; count can be set."""
    from paper_2609_32415_gb300 import RefAdaptError
    t = training()
    base = torch.arange(150.0, device="cuda")
    params = [torch.nn.Parameter(base[:100]), torch.nn.Parameter(base[50:])]
    opt = t.AdamW(params, 1e-2, capturable=capturable)
    opt.count = 5
    for p in params:
        p.grad = torch.ones_like(p)
    with pytest.raises(RefAdaptError, match="overlaps"):
        opt.step()
    assert int(opt.count) == 5 and torch.equal(base, torch.arange(150.0, device="cuda"))
    other = t.AdamW(params[:1], 1e-2, capturable=not capturable)
    other.load_state_dict({**other.state_dict(), "count": opt.count})
    assert int(other.count) == 5


def test_linear4_difference_along_the_gradient(cuda_ok):
    """Along its own gradient G = up W (and up^T x for the weight) the loss changes by step |G|. 4 bits change that by
    the operands' errors, together below 0.2 of |G| normwise (test_gpu_linear4_layers derives it), and each of the two
    losses by at most 0.2 |G| rms(x): beside a step of 64 that is 0.01. The gradient that came back, 0.2 off G at most, along the same
    step likewise. A gradient of zero or of the wrong sign is 1 or 2 off."""
    t4, g = training().linear4, torch.Generator().manual_seed(33)
    x, w, up = (torch.randn(s, generator=g).mul(k).to(torch.bfloat16).cuda()
                for s, k in (((1, 256, 256), 1.0), ((256, 256), 0.06), ((1, 256, 256), 1.0)))
    xr, wr = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    (t4(xr, wr) * up).float().sum().backward()

    def loss(x, w):
        return float((t4(x.to(torch.bfloat16), w.to(torch.bfloat16)).double() * up.double()).sum())

    for i, (t, got, G) in enumerate(((x, xr.grad, up.double() @ w.double()), (w, wr.grad, up[0].double().T @ x[0].double()))):
        size = float(G.norm())
        length = 64.0 if i == 0 else 64.0 * 0.06
        step = G / size * length
        a, b = ((t.double() + s * step) for s in (0.5, -0.5))
        moved = loss(a, w) - loss(b, w) if i == 0 else loss(x, a) - loss(x, b)
        assert abs(moved - length * size) < 0.22 * length * size
        assert abs(float((got.double() * step).sum()) - length * size) < 0.2 * length * size
