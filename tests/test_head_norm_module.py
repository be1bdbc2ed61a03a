"""MSHeadNormRotary in models that change their type: its frequencies stay as they were made
(no GPU: the library's calls are noted, not made)."""
import pytest
import torch
from torch import nn

from paper_2404_12406_amd import api
from paper_2404_12406_amd import autograd as msa

FREQ = api.rotary_frequencies(64)


@pytest.fixture
def specs(monkeypatch):
    seen = []

    def layer_forward(spec, x, W=None, b=None, mask=0, y=None):
        seen.append((spec, W))
        return torch.zeros_like(x), None

    monkeypatch.setattr(api, "layer_forward", layer_forward)
    return seen


CONVERT = {"bf16": lambda m: m.bfloat16(), "to": lambda m: m.to(torch.bfloat16), "there and back": lambda m: m.bfloat16().float(),
           "64 bits": lambda m: m.double(), "with the device": lambda m: m.to("cpu", torch.bfloat16), "half": lambda m: m.half().bfloat16()}


@pytest.mark.parametrize("how", CONVERT)
@pytest.mark.parametrize("norm", [True, False])
def test_frequencies_keep_their_type(norm, how, specs):
    w = torch.rand(64) if norm else None
    model = nn.Sequential(nn.Linear(4, 4), msa.MSHeadNormRotary(w, w, 2, FREQ.clone(), norm=norm))
    model = CONVERT[how](model)
    m = model[1]
    assert m.inv_freq.dtype == torch.float32 and torch.equal(m.inv_freq, FREQ)
    x = torch.randn(3, 4, 64, dtype=model[0].weight.dtype)
    with torch.no_grad():
        m(x, torch.arange(3, dtype=torch.int32))
    spec, W = specs.pop()
    assert torch.equal(spec.inv_freq, FREQ) and spec.inv_freq.dtype == torch.float32
    assert W is None or W.dtype == x.dtype
    assert not [k for k in model.state_dict() if "freq" in k]


def test_frequencies_follow_the_device():
    m = msa.MSHeadNormRotary(None, None, 2, FREQ.clone(), norm=False)
    m = m.to(device="meta", dtype=torch.bfloat16)
    assert m.inv_freq.device.type == "meta" and m.inv_freq.dtype == torch.float32


def test_modules_without_frequencies_convert():
    m = msa.MSHeadNormRotary(torch.rand(8), None, 2).bfloat16()
    assert m.inv_freq is None and m.weight_q.dtype == torch.bfloat16


@pytest.mark.parametrize("mode", [torch.no_grad, torch.enable_grad])
def test_frequencies_without_positions_are_refused(mode, monkeypatch):
    """As by the layer itself: nothing is computed without the rotation that the module describes."""
    made = []
    monkeypatch.setattr(api, "_one_gpu", lambda *a: None)
    monkeypatch.setattr(api, "_block_run", lambda *a: made.append(a) or 0)
    monkeypatch.setattr(api, "_stream", lambda d: None)
    w = torch.rand(64)
    for m in (msa.MSHeadNormRotary(w, w, 2, FREQ), msa.MSHeadNormRotary(None, None, 2, FREQ, norm=False)):
        with mode(), pytest.raises(ValueError, match="without positions"):
            m(torch.randn(3, 4, 64))
    assert not made
    with torch.no_grad():   # a module without frequencies needs none
        assert msa.MSHeadNormRotary(w, w, 2)(torch.randn(3, 4, 64)).shape == (3, 4, 64)
    assert len(made) == 1
