"""What training.AdamW and training.linear4 leave behind in torch's graph and in their own state."""
import pytest
import torch

from test_gpu_linear4 import bf

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
