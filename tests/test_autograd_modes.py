"""What the modules ask of the library by grad mode (no GPU: the library's calls are
noted, not made): where no gradient can be taken, nothing is kept for one."""
import pytest
import torch

from paper_2404_12406_amd import api
from paper_2404_12406_amd import autograd as msa

P = lambda *s: torch.randn(*s)
CL = lambda *s: torch.randn(*s).contiguous(memory_format=torch.channels_last)

MODULES = {
    "norm": (lambda: msa.MSLayerNorm(P(8), P(8)), lambda: (P(3, 8),), 7),
    "gated": (lambda: msa.MSGatedLinear(P(12, 8), P(12)), lambda: (P(3, 8),), 7),
    "xent": (lambda: msa.MSLinearCrossEntropy(P(11, 8), P(11)), lambda: (P(3, 8), torch.tensor([1, 2, 3])), 7),
    "linear": (lambda: msa.MSLinear(P(6, 8), P(6)), lambda: (P(3, 8),), 7),
    "conv": (lambda: msa.MSConv2d(CL(4, 3, 3, 3), P(4), 1, 1), lambda: (CL(2, 3, 5, 5),), 7),
    "bn": (lambda: msa.MSBatchNorm2dEval(P(3), P(3), P(3), P(3).abs()), lambda: (CL(2, 3, 5, 5),), 7),
    "relu": (lambda: msa.MSReLU(), lambda: (P(3, 8),), 1),
    "dropout": (lambda: msa.MSDropout(0.5), lambda: (P(3, 8),), 1),
}


class Kept:
    """Stands for a record that borrows the layer's input."""

    def __init__(self, x):
        self.saved = {"x": x}

    def free(self):
        pass


@pytest.fixture
def masks(monkeypatch):
    seen = []

    def layer_forward(spec, x, W=None, b=None, mask=0, y=None):
        seen.append(mask)
        return torch.zeros(api.output_shape(spec, x, W)), (Kept(x) if mask else None)

    monkeypatch.setattr(api, "layer_forward", layer_forward)
    return seen


@pytest.mark.parametrize("name", MODULES)
def test_modules_keep_nothing_without_grad_mode(name, masks):
    make, inputs, full = MODULES[name]
    m, args = make(), inputs()
    args[0].requires_grad_()
    with torch.no_grad():
        want = m(*args).shape
    assert masks == [0]
    y = m(*args)
    assert y.requires_grad and y.shape == want and masks == [0, full]
    m.requires_grad_(False)
    m(args[0].detach(), *args[1:])
    assert masks == [0, full, 0]


@pytest.mark.parametrize("name", MODULES)
def test_modules_run_in_inference_mode(name, masks):
    make, inputs, _ = MODULES[name]
    m = make()   # with parameters that train
    with torch.inference_mode():
        y = m(*inputs())
    assert not y.requires_grad and masks == [0]


@pytest.mark.parametrize("name", MODULES)
def test_a_second_backward_is_refused(name, masks, monkeypatch):
    """The first consumes the record; a graph that is retained has no second gradient to give."""
    def layer_backward(rec, gy, *buffers):
        return tuple(torch.zeros_like(t) if t is not None else None for t in rec.grads)

    make, inputs, _ = MODULES[name]
    m, args = make(), inputs()
    x = args[0].requires_grad_()
    monkeypatch.setattr(api, "layer_backward", layer_backward)
    shapes = (x.reshape(-1, x.shape[-1]) if x.dim() == 2 else x, getattr(m, "weight", None), getattr(m, "bias", None))
    monkeypatch.setattr(Kept, "grads", shapes, raising=False)
    loss = m(*args).sum()
    loss.backward(retain_graph=True)
    assert x.grad is not None
    with pytest.raises(RuntimeError, match="second time"):
        loss.backward()
