"""What a record borrows, when its backward runs on another stream than its forward (no
GPU: streams and the library's calls are stand-ins)."""
import ctypes

import pytest
import torch

from paper_2404_12406_amd import api


class Tensor:
    """Notes the streams that its memory must outlive."""

    def __init__(self):
        self.streams = []

    def record_stream(self, s):
        self.streams.append(s)


class Lib:
    def ms_record_account(self, h, acct):
        acct._obj.mask, acct._obj.borrowed = 3, 3
        return 0

    def ms_layer_backward(self, *a):
        return 0

    def ms_record_free(self, h):
        return 0


@pytest.fixture
def stream(monkeypatch):
    """Sets the current stream."""
    current = [11]
    monkeypatch.setattr(api._lib, "load", lambda: Lib())
    monkeypatch.setattr(api, "_stream", lambda device: ctypes.c_void_p(current[0]))
    monkeypatch.setattr(api, "_block_fn", lambda name: lambda *a: 0)
    monkeypatch.setattr(api, "_one_gpu", lambda *t: None)
    monkeypatch.setattr(api, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    return lambda s: current.__setitem__(0, s)


@pytest.fixture
def record(stream):
    """api.Record(...) of a handle that no library knows."""
    made = []

    def make(*args, **kw):
        made.append(api.Record(ctypes.c_void_p(1), *args, **kw))
        return made[-1]

    yield make
    for rec in made:
        rec._h = None


@pytest.mark.parametrize("spec", [api.GatedLinear(), api.Linear(), api.ReLU()], ids=["gated", "linear", "relu"])
def test_borrowed_memory_outlives_a_backward_on_another_stream(stream, record, spec):
    x, W = torch.zeros(4, 8), torch.zeros(6, 8)
    for back, want in ((11, []), (22, [22])):
        stream(11)
        block = not isinstance(spec, (api.Linear, api.ReLU))
        rec = record(api._BlockDesc(spec) if block else api._LayerDesc(spec), x, W, None, (4, 6), x)
        kept = {"x": Tensor(), "W": Tensor(), "stats": (Tensor(), Tensor()), "projections": Tensor()}
        rec._keep = dict(kept)
        stream(back)
        api.layer_backward(rec, torch.zeros(4, 8))
        for t in (kept["x"], kept["W"], *kept["stats"], kept["projections"]):
            assert t.streams == want
        assert rec.consumed and not rec.saved


def test_a_kept_gradient_holds_no_targets(record):
    """(8 bytes a row, and what they are a view of.)"""
    import weakref
    t = torch.zeros(4, dtype=torch.int64)
    gone = weakref.ref(t)
    spec = api.LinearCrossEntropy(t)
    rec = record(api._BlockDesc(spec), torch.zeros(4, 8), torch.zeros(6, 8), None, (1,), t, extra={"grad": Tensor()})
    del t, spec
    assert gone() is None and "grad" in rec.saved
