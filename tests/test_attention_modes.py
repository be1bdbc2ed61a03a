"""What attention's modules ask of the library by grad mode, and what the Python entry points
refuse before they call it (no GPU: the library's calls are noted, not made)."""
import pytest
import torch

from paper_2404_12406_amd import api
from paper_2404_12406_amd import autograd as msa

P = lambda *s: torch.randn(*s)
I = lambda *v: torch.tensor(v, dtype=torch.int32)
FREQ = api.rotary_frequencies(8)


# ------------------------------------------------------------------ modules
def rotary(x):
    return msa.MSHeadNormRotary(P(8), P(8), 2, FREQ), (x, I(0, 1, 2))


def turned(x):
    return msa.MSHeadNormRotary(None, None, 2, FREQ, norm=False), (x, I(0, 1, 2))


def normed(x):
    return msa.MSHeadNormRotary(P(8), None, 2), (x,)


# the module and its arguments, its mask with every parameter and input that trains
MODULES = {"rotary": (rotary, 7), "turned": (turned, 1), "normed": (normed, 3)}


class Kept:
    """Stands for a record that borrows the layer's input."""

    def __init__(self, x):
        self.saved = {"x": x}

    def free(self):
        pass


@pytest.fixture
def seen(monkeypatch):
    calls = []

    def layer_forward(spec, x, W=None, b=None, mask=0, y=None):
        calls.append((spec, mask))
        return torch.zeros(api.output_shape(spec, x, W)), (Kept(x) if mask else None)

    monkeypatch.setattr(api, "layer_forward", layer_forward)
    return calls


@pytest.mark.parametrize("name", MODULES)
def test_head_norms_keep_nothing_without_grad_mode(name, seen):
    make, full = MODULES[name]
    x = P(3, 4, 8).requires_grad_()
    m, args = make(x)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert m(*args).shape == x.shape
        assert seen.pop()[1] == 0
    y = m(*args)
    assert y.requires_grad and y.shape == x.shape and seen.pop()[1] == full
    m.requires_grad_(False)
    m(x.detach(), *args[1:])
    assert seen.pop()[1] == 0
    m(*args)
    assert seen.pop()[1] == 1


@pytest.mark.parametrize("mask", range(8))
def test_attention_asks_for_the_gradients_that_are_wanted(mask, seen):
    q, k, v = (P(*s).requires_grad_(bool(mask >> i & 1)) for i, s in enumerate(((3, 4, 8), (5, 2, 8), (5, 2, 8))))
    m = msa.MSAttention(causal=False, scale=0.5)
    off, k_off = I(0, 1, 3), I(0, 4, 5)
    assert m(q, k, v, off, k_off).requires_grad == (mask > 0)
    spec, got = seen.pop()
    assert got == mask and spec == api.Attention(off, k_off, False, 0.5)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            m(q, k, v)
        assert seen.pop()[1] == 0


def test_parameters_and_buffers():
    m = msa.MSHeadNormRotary(P(8), P(8), 2, FREQ)
    assert set(m.state_dict()) == {"weight_q", "weight_k"}   # the frequencies follow from the model's description
    assert m.to(torch.bfloat16).weight_q.dtype == torch.bfloat16
    p = torch.nn.Parameter(P(8))
    assert msa.MSHeadNormRotary(p, p, 2).weight_k is p       # one scale for queries and keys


@pytest.mark.parametrize("dim,theta", [(2, 10000.0), (64, 10000.0), (128, 5e5)])
def test_frequencies(dim, theta):
    want = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    f = api.rotary_frequencies(dim, theta)
    assert f.dtype == torch.float32 and f.shape == (dim // 2,)
    assert torch.equal(f, want.float()) or (f.double() / want - 1).abs().max() <= 2 ** -23


# ------------------------------------------------------------------ refusals
@pytest.fixture
def calls(monkeypatch):
    made = []

    class Fns(dict):
        def get(self, name, default=None):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(api, "_one_gpu", lambda *a: None)
    monkeypatch.setattr(api, "_stream", lambda d: None)
    monkeypatch.setattr(api, "_block_fns", Fns())
    return made


Q, K_, V_ = P(3, 4, 8), P(3, 2, 8), P(3, 2, 8)
PAGES, TAB, LEN = P(5, 2, 4, 8), I(0, 1, 2, 3, 4, 0).reshape(3, 2), I(1, 2, 3)
X = P(3, 8, 8)


def cache(**over):
    return dict(dict(k_pages=PAGES, v_pages=PAGES, tables=TAB), **over)


GOOD = {
    "rotary": lambda **o: (api.HeadNormRotary(**{**dict(positions=LEN, inv_freq=FREQ, q_heads=2), **o}), X, P(8), P(8)),
    "attention": lambda **o: (api.Attention(**{**dict(offsets=I(0, 1, 3)), **o}), Q, K_, V_),
    "append": lambda **o: (api.CacheAppend(**{**cache(positions=LEN, inv_freq=FREQ, q_heads=4), **o}), X, P(8), P(8)),
    "paged": lambda **o: (api.PagedAttention(**{**cache(lengths=LEN), **o}), Q),
}
BAD = [(k, TypeError, o) for k in ("rotary", "append") for o in (
    dict(positions=LEN.long()), dict(inv_freq=FREQ.double()), dict(inv_freq=FREQ.reshape(2, 2)), dict(inv_freq=P(8)[::2]))] + [
    (k, ValueError, dict(positions=I(0, 1))) for k in ("rotary", "append")] + [
    ("rotary", ValueError, dict(positions=None)), ("append", ValueError, dict(positions=None)),
    ("rotary", ValueError, dict(positions=I(0, 0, 1, 0, 2, 0)[::2])),
    ("attention", TypeError, dict(offsets=I(0, 1, 3).long())), ("attention", ValueError, dict(offsets=I(0, 3).reshape(1, 2))),
    ("attention", ValueError, dict(offsets=I())), ("attention", ValueError, dict(offsets=None, k_offsets=I(0, 1, 3))),
    ("attention", ValueError, dict(k_offsets=I(0, 3))), ("attention", TypeError, dict(k_offsets=I(0, 1, 3).long())),
] + [(k, e, o) for k in ("append", "paged") for e, o in (
    (TypeError, dict(tables=TAB.long())), (ValueError, dict(tables=TAB.reshape(-1))), (ValueError, dict(tables=TAB.t())),
    (ValueError, dict(k_pages=PAGES[0])), (TypeError, dict(v_pages=PAGES.half())))] + [
    ("append", TypeError, dict(rows=LEN.long())), ("append", ValueError, dict(rows=I(0, 1))),
    ("paged", TypeError, dict(lengths=LEN.long())), ("paged", ValueError, dict(lengths=I(1, 2))), ("paged", ValueError, dict(lengths=LEN[:, None])),
]


@pytest.mark.parametrize("kind", GOOD)
def test_calls_that_are_made(kind, calls):
    y, rec = api.layer_forward(*GOOD[kind]())
    assert rec is None and y.shape == (3, {"rotary": 8}.get(kind, 4), 8) and len(calls) == 1


@pytest.mark.parametrize("kind,error,over", BAD)
def test_arguments_that_are_refused(kind, error, over, calls):
    with pytest.raises(error):
        api.layer_forward(*GOOD[kind](**over))
    assert not calls


@pytest.mark.parametrize("kind", GOOD)
def test_tensors_that_are_refused(kind, calls):
    spec, x, *rest = GOOD[kind]()
    for bad, error in ((x[0], ValueError), (x.half(), TypeError), (x.double(), TypeError)):
        with pytest.raises(error):
            api.layer_forward(spec, bad, *rest)
    if kind == "attention":
        for bad in ((None, V_), (K_, None), (K_[0], V_)):
            with pytest.raises(TypeError):
                api.layer_forward(spec, x, *bad)
    if kind == "paged":
        with pytest.raises(TypeError):
            api.layer_forward(spec, x, P(8))
    assert not calls


@pytest.mark.parametrize("kind", ["append", "paged"])
def test_serving_layers_have_no_gradients(kind, calls):
    with pytest.raises(ValueError, match="no gradients"):
        api.layer_forward(*GOOD[kind](), mask=1)
    assert not calls


def test_tensors_elsewhere_are_refused():
    """(The CPU is no GPU.)"""
    for kind in GOOD:
        with pytest.raises(TypeError, match="on the GPU only"):
            api.layer_forward(*GOOD[kind]())
