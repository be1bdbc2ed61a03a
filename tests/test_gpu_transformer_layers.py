"""The transformer layers as a program uses them: every tile their contractions
may take, captured and replayed, backward without allocation, without memory
for their workspace, and together in the fine-tuning example against the same
model in 64 bits."""
import ctypes
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import _lib
from paper_2404_12406_amd.api import _ptr, _stream, tensor_desc
from _gpu import TORCH_DT, check, host

import test_gpu_gated_linear as gated
import test_gpu_layer_norm as norm
import test_gpu_linear_cross_entropy as xent

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------ tiles
@pytest.fixture
def tile(request, monkeypatch):
    monkeypatch.setenv("MEMSAVE_FUSED_TILE", request.param)
    return request.param


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("shape", [(300, 264, 200), (515, 1000, 66)])
@pytest.mark.parametrize("tile", ["256x256", "128x128", "128x128s4"], indirect=True)
def test_gated_tiles(tile, shape, keep):
    t = gated.inputs(*shape, "bf16")
    gated.compare(gated.run(*gated.cuda(*t), "gelu", keep, 7), t, "gelu", 7, "bf16")


@pytest.mark.parametrize("shape", [(300, 264, 1000), (515, 520, 2050), (70, 1000, 515)])
@pytest.mark.parametrize("tile", ["256x256", "256x128", "128x128", "128x128s4", "128x128w8"], indirect=True)
def test_cross_entropy_tiles(tile, shape):
    t = xent.inputs(*shape, "bf16", ignored=0.3)
    xent.compare(xent.run(*xent.cuda(*t), "mean", 7), t, "mean", 7, "bf16")


# ------------------------------------------------------------------ layers of one call
def layer(kind, M, D, dtype, seed=0):
    """(spec, x, W, b, gradient of the output) on the GPU."""
    if kind == "norm":
        x, g, b, dy = norm.inputs(M, D, dtype, seed)
        return (ms.LayerNorm(1e-5),) + tuple(t.cuda() for t in (x, g, b, dy))
    if kind.startswith("gated"):
        x, W, b, dy = gated.inputs(M, D, 200, dtype, seed=seed)
        spec = ms.GatedLinear("silu", "projections" if kind == "gated" else "input")
        return (spec,) + gated.cuda(x, W, b, dy)
    x, W, b, t, gl = xent.inputs(M, D, 1000, dtype, ignored=0.2, seed=seed)
    return ms.LinearCrossEntropy(t.cuda()), x.cuda(), W.cuda(), b.cuda(), gl.cuda()


KINDS = ["norm", "gated", "gated_input", "xent"]


def passes(spec, x, W, b, dy):
    y, rec = ms.layer_forward(spec, x, W, b, 7)
    return (y,) + ms.layer_backward(rec, dy)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [4, 300])
@pytest.mark.parametrize("kind", KINDS)
def test_replays_of_a_graph(kind, M, dtype):
    """Widths that need padded copies among them; new inputs between the replays,
    and other work on the stream that outgrows the captured workspace."""
    for D in (264, 515):
        args = layer(kind, M, D, dtype)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            passes(*args)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = passes(*args)
        for i in range(3):
            other = layer(kind, M, D, dtype, seed=100 + i)
            for into, new in zip(args[1:], other[1:]):
                into.copy_(new)
            if kind == "xent":
                args[0].target.copy_(other[0].target)
            for t in got:
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in got]
            with torch.cuda.stream(stream):
                want = passes(*args)
                passes(*layer("xent", 700 + 100 * i, 515, dtype))
            torch.cuda.synchronize()
            for a, c in zip(replayed, want):
                assert not torch.isnan(a.float()).any()
                assert torch.equal(a, c), (kind, D, i)


def c_backward(entry, rec, dy, x, W, b):
    outs = [torch.full_like(t, float("nan")) for t in (x, W, b)]
    st = getattr(_lib.load(), entry)(rec._h, _ptr(tensor_desc(dy)), *(_ptr(tensor_desc(t)) for t in outs), _stream(x.device))
    torch.cuda.synchronize()
    return st, outs


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_backward_without_allocation(kind, dtype):
    for M, D in ((300, 264), (70, 515)):
        spec, x, W, b, dy = layer(kind, M, D, dtype)
        outs = []
        for entry in ("ms_layer_backward", "ms_layer_backward_noalloc"):
            _, rec = ms.layer_forward(spec, x, W, b, 7)
            assert rec.account()["transient_workspace_bytes"] <= _lib.load().ms_noalloc_scratch_bytes()
            st, got = c_backward(entry, rec, dy, x, W, b)
            assert st == 0, _lib.load().ms_last_error().decode()
            outs.append(got)
            rec.free()
        for a, c in zip(*outs):
            assert not torch.isnan(a.float()).any() and torch.equal(a, c)


def test_backward_beyond_the_fixed_scratch_is_refused():
    dy = torch.ones(1, device="cuda")
    W = torch.zeros(200000, 264, dtype=torch.bfloat16, device="cuda")   # dz of 2048 rows alone has 819 MB
    b = torch.zeros(200000, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(2048, 264, device="cuda").bfloat16()
    spec = ms.LinearCrossEntropy(torch.zeros(2048, dtype=torch.int64, device="cuda"))
    _, rec = ms.layer_forward(spec, x, W, b, 7)
    assert rec.account()["transient_workspace_bytes"] > _lib.load().ms_noalloc_scratch_bytes()
    live = ms.ledger_read()[0]
    st, outs = c_backward("ms_layer_backward_noalloc", rec, dy, x, W, b)
    assert st == _lib.MS_E_UNSUPPORTED and all(bool(torch.isnan(t.float()).all()) for t in outs)
    assert ms.ledger_read()[0] == live
    st, outs = c_backward("ms_layer_backward", rec, dy, x, W, b)
    assert st == 0 and not any(bool(torch.isnan(t.float()).any()) for t in outs)
    rec.free()


@pytest.mark.parametrize("kind", KINDS)
def test_without_memory_for_the_workspace(kind):
    """Refused before anything runs; the record stays usable."""
    lib = _lib.load()
    spec, x, W, b, dy = layer(kind, 300, 515, "bf16")
    _, rec = ms.layer_forward(spec, x, W, b, 7)
    live = ms.ledger_read()[0]
    torch.cuda.synchronize()
    handle = ctypes.c_void_p()   # a stream that has no workspace yet: torch's are handed out again
    assert lib.hipStreamCreate(ctypes.byref(handle)) == 0
    with torch.cuda.stream(torch.cuda.ExternalStream(handle.value)):
        lib.ms_testing_fail_next_workspace(1)
        st, outs = c_backward("ms_layer_backward", rec, dy, x, W, b)
        lib.ms_testing_fail_next_workspace(0)
    assert st == _lib.MS_E_NOMEM and all(bool(torch.isnan(t.float()).all()) for t in outs)
    assert ms.ledger_read()[0] == live
    st, outs = c_backward("ms_layer_backward", rec, dy, x, W, b)
    assert st == 0 and not any(bool(torch.isnan(t.float()).any()) for t in outs)
    rec.free()


# ------------------------------------------------------------------ the example
@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("finetune_example", os.path.join(ROOT, "examples", "finetune.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def reference(model, tokens, targets, act):
    """(loss, {parameter: gradient}) of the same model in 64 bits."""
    p = {n: v.detach().double().cpu().requires_grad_(v.requires_grad) for n, v in model.named_parameters()}
    F = torch.nn.functional
    fn = {"silu": F.silu, "gelu": F.gelu}[act]
    x = p["embed"][tokens]
    for i in range(len(model.blocks)):
        q = {n.split(".", 2)[2]: v for n, v in p.items() if n.startswith(f"blocks.{i}.")}
        h = F.layer_norm(x, x.shape[-1:], q["norm.weight"], q["norm.bias"])
        g, u = F.linear(h, q["gate.weight"], q["gate.bias"]).chunk(2, -1)
        x = x + F.linear(fn(g) * u, q["down.weight"], q["down.bias"])
    x = F.layer_norm(x, x.shape[-1:], p["norm.weight"], p["norm.bias"])
    loss = F.cross_entropy(F.linear(x, p["head.weight"]), targets, ignore_index=-100)
    loss.backward()
    return loss.item(), {n: v.grad for n, v in p.items() if v.grad is not None}


@pytest.mark.parametrize("what", ["all", "norms"])
@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_gradients(example, dtype, keep, what):
    """Bars: fp32 sums of at most some 1e4 terms through ten layers, 1e-4.  bf16:
    some ten layers, each rounding its output and its gradient (2^-9 each, of
    errors that add up as a root: 2^-7), where an element's worst is some four times
    the usual: 2^-5."""
    model = example.NextToken(words=1003, width=136, hidden=347, act="gelu", keep=keep, dtype=TORCH_DT[dtype]).train_only(what)
    g = torch.Generator().manual_seed(5)
    tokens = torch.randint(0, 1003, (333,), generator=g)
    targets = torch.randint(0, 1003, (333,), generator=g)
    targets[::5] = -100
    loss = model(tokens.cuda(), targets.cuda())
    loss.backward()
    want, grads = reference(model, tokens, targets, "gelu")
    bar = {"f32": 1e-4, "bf16": 2.0 ** -5}[dtype]
    check("loss", np.array([loss.item()]), np.array([want]), dtype, bar)
    got = {n: v.grad for n, v in model.named_parameters() if v.grad is not None}
    assert got.keys() == grads.keys() and len(got) == (2 * 6 + 4 if what == "all" else 2 * 2 + 2)
    for n, v in got.items():
        check(n, host(v), grads[n].numpy(), dtype, bar)
    assert ms.ledger_read()[0] == 0


def test_example_learns_and_scores(example):
    lines = []
    model = example.NextToken(words=256, width=128, hidden=128)
    losses, follows = example.train(model, steps=60, batch=1024, rate=1e-2, report=lines.append)
    assert losses[-1] < 0.5 * losses[0] and len(lines) == 60
    tokens = torch.arange(256)
    with torch.no_grad():
        mean = model(tokens.cuda(), follows.cuda())
    scores = torch.cat([model.score(tokens[i:i + 1].cuda(), follows[i:i + 1].cuda()) for i in range(8)])
    many = model.score(tokens.cuda(), follows.cuda())
    # a token alone takes another split of the same fp32 sums: its bf16 hidden states may round apart
    assert torch.allclose(scores, many[:8], atol=0.05)
    assert abs(many.mean().item() + mean.item()) < 1e-4
    assert ms.ledger_read()[0] == 0
