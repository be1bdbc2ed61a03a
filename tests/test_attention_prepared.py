"""A prepared call holds every tensor it describes, whatever becomes of its description (no GPU)."""
import gc
import weakref

import pytest
import torch

from paper_2404_12406_amd import api

I = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731


def specs():
    pages = [torch.zeros(5, 2, 4, 8) for _ in range(2)]
    tables, freq = I(0, 1, 2, 3, 4, 0).reshape(3, 2), api.rotary_frequencies(8)
    x = torch.zeros
    return {
        "rotary": (api.HeadNormRotary(I(0, 1, 2), freq, 2), x(3, 4, 8), x(8), x(8)),
        "attention": (api.Attention(I(0, 1, 3), I(0, 1, 3)), x(3, 4, 8), x(3, 2, 8), x(3, 2, 8)),
        "append": (api.CacheAppend(*pages, tables, I(0, 1, 2), I(0, 1, 2), freq, 4), x(3, 8, 8), x(8), x(8)),
        "paged": (api.PagedAttention(*pages, tables, I(1, 2, 3)), x(3, 4, 8)),
    }


@pytest.mark.parametrize("kind,mask", [("rotary", 0), ("rotary", 7), ("attention", 0), ("attention", 4), ("attention", 7), ("append", 0), ("paged", 0)])
def test_tensors_of_a_changed_description_live_on(kind, mask, monkeypatch):
    monkeypatch.setattr(api, "_one_gpu", lambda *a: None)
    monkeypatch.setattr(api, "_on_gpu", lambda *a: None)
    monkeypatch.setattr(api, "_stream", lambda d: None)
    spec, *tensors = specs()[kind]
    call = api.PreparedLayer(spec, *tensors, mask=mask)
    fields = [(n, weakref.ref(v)) for n, v in vars(spec).items() if isinstance(v, torch.Tensor)]
    assert len(fields) >= 2
    for n, _ in fields:
        setattr(spec, n, None)   # as a program that prepares its next call with the same object
    gc.collect()
    assert not [n for n, r in fields if r() is None]
    del call
    gc.collect()
    assert not [n for n, r in fields if r() is not None]
