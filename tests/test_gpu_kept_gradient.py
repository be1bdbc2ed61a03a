"""Cross entropy of a frozen head, whose forward takes the input's gradient, against
the formulas in 64 bits.

Bars: those of test_gpu_linear_cross_entropy.py.  The exponentials are rounded to
bf16 once (2^-9, averaging out over the words), the target's part of dx is not
rounded before the result; the kept 24 bits add 2^-17."""
import numpy as np
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import TORCH_DT, check, host

from test_gpu_linear_cross_entropy import BAR, IGNORE, LOSS, draw, inputs

pytestmark = pytest.mark.gpu


def reference(x, W, b, t, gl, reduction, ignore=IGNORE):
    """(loss, dx) on the GPU, in 64 bits, 1024 rows at a time."""
    live = (t != ignore).nonzero()[:, 0]
    each, dx = torch.zeros(len(t), dtype=torch.float64, device="cuda"), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    g = gl.double() if reduction == "none" else gl.double().expand(len(t)) / (len(live) if reduction == "mean" else 1)
    Wd = W.double()
    for rows in live.split(1024):
        z = x[rows].double() @ Wd.t()
        if b is not None:
            z += b.double()
        lse = torch.logsumexp(z, 1)
        k = torch.arange(len(rows), device="cuda")
        each[rows] = lse - z[k, t[rows]]
        dz = torch.exp(z - lse[:, None])
        dz[k, t[rows]] -= 1
        dx[rows] = (dz * g[rows, None]) @ Wd
    loss = each if reduction == "none" else each.sum()[None] / (len(live) if reduction == "mean" else 1)
    return loss, dx


def run(x, W, b, t, gl, reduction="mean", ignore=IGNORE):
    loss, rec = ms.layer_forward(ms.LinearCrossEntropy(t, ignore, reduction), x, W, b, 1)
    assert set(rec.saved) == {"grad"}   # the path under test
    return loss, ms.layer_backward(rec, gl)[0]


def compare(outs, t, reduction, dtype, largest=0.0):
    """`largest`: the logits' size where that is more than some tens; their own errors,
    2^-23 of it, are then those of the exponentials (twice that is allowed)."""
    loss, dx = reference(*t, reduction)
    check("loss", host(outs[0]), host(loss), "f32", LOSS)
    check("dx", host(outs[1]), dx.cpu().numpy(), dtype, BAR[dtype] + largest * 2.0 ** -22)


def cuda(*ts):
    return tuple(None if v is None else v.cuda() for v in ts)


# just past the few-row kernels, ragged rows, widths, vocabularies, long ones
SHAPES = [(17, 1000, 130001), (300, 264, 30000), (515, 130, 40003), (1030, 515, 5001), (4097, 64, 9000), (2050, 2056, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    t = cuda(*inputs(*shape, dtype))
    compare(run(*t), t, "mean", dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("ignored", [0.0, 0.4, 0.95])
def test_reductions_and_ignored_rows(ignored, reduction, dtype):
    t = cuda(*inputs(400, 200, 30000, dtype, ignored != 0.4, ignored, reduction, 11))
    compare(run(*t, reduction), t, reduction, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_every_row_ignored(reduction, dtype):
    x, W, b, t, gl = cuda(*inputs(400, 200, 30000, dtype, reduction=reduction, seed=21))
    loss, dx = run(x, W, b, torch.full_like(t, IGNORE), gl, reduction)
    assert torch.isnan(loss).all() if reduction == "mean" else bool((loss == 0).all())
    assert bool((dx == 0).all())


@pytest.mark.parametrize("std", [0.01, 30.0, 1000.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes_of_logits(dtype, std):
    """From nearly none to rows whose parts are hundreds of powers of two apart."""
    x, W, b, t, gl = inputs(300, 264, 30000, dtype, seed=31)
    t = cuda((x.float() * std / 3).to(x.dtype), W, b, t, gl)
    compare(run(*t), t, "mean", dtype, 5 * std)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_confident_rows(dtype):
    """Targets that have nearly all of the probability, in part to within rounding."""
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, False, seed=41))
    Wt = W[t].float()
    for most in (40, 6):   # the second: the least confident alone
        x = (Wt * (torch.linspace(2, most, 300, device="cuda")[:, None] / (Wt * Wt).sum(1, keepdim=True))).to(W.dtype)
        args = (x, W, b, t, gl)
        compare(run(*args), args, "mean", dtype)


@pytest.mark.parametrize("low", [-float("inf"), -3e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_words(dtype, low):
    """Words left out by their bias, whole column tiles among them."""
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, seed=51))
    b[:1000] = low
    b[2000:] = low
    t = 1000 + t % 1000
    got = run(x, W, b, t, gl)
    keep = slice(1000, 2000)
    loss, dx = reference(x, W[keep], b[keep], t - 1000, gl, "mean")
    check("loss", host(got[0]), host(loss), "f32", LOSS)
    check("dx", host(got[1]), dx.cpu().numpy(), dtype, BAR[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_far_apart(dtype):
    """Groups of words hundreds below and above the others, and a target among the low ones."""
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, seed=61))
    b += (torch.arange(30000, device="cuda") // 100 % 7 * 60.0 - 180.0).to(b.dtype)
    t = (x, W, b, t, gl)
    compare(run(*t), t, "mean", dtype, 200.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_word_of_the_lowest_value(dtype):
    """A distribution, if an even one: nothing but the common value is lost."""
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, seed=71))
    b[:] = -3e38
    loss, dx = run(x, W, b, t, gl, "sum")
    p = 1.0 / 30000
    want = (p * W.double().sum(0) - W[t].double()) * gl.double()
    check("loss", host(loss), np.array([300 * np.log(30000)]), "f32", LOSS)
    check("dx", host(dx), want.cpu().numpy(), dtype, BAR[dtype])
    b[:] = -float("inf")
    loss, dx = run(x, W, b, t, gl, "sum")
    assert torch.isnan(loss).all() and torch.isnan(dx.float()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_rows_stay_in_their_rows(dtype):
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, True, 0.0, "none", 81))
    want = reference(x, W, b, t, gl, "none")
    t = t.clone()
    x[3, 5], x[70, 0], x[200, 263] = float("nan"), float("inf"), -float("inf")
    t[9], t[10], t[11], t[12] = 30000, -1, 2 ** 40, IGNORE
    x[12] = float("nan")
    loss, dx = run(x, W, b, t, gl, "none")
    bad = [3, 70, 200, 9, 10, 11]
    assert torch.isnan(loss[bad]).all() and torch.isnan(dx[bad].float()).any(1).all()
    assert loss[12] == 0 and bool((dx[12] == 0).all())
    ok = [i for i in range(300) if i not in bad and i != 12]
    check("loss", host(loss[ok]), host(want[0][ok]), "f32", LOSS)
    check("dx", host(dx[ok]), want[1][ok].cpu().numpy(), dtype, BAR[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_masked_target(dtype):
    """An infinite loss; its gradient is that of the others' softmax less the target's word."""
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, dtype, True, 0.0, "none", 91))
    want = reference(x, W, b, t, gl, "none")
    b = b.clone()
    t[7] = 123
    b[123] = -float("inf")
    loss, dx = run(x, W, b, t, gl, "none")
    assert loss[7] == float("inf") and bool(torch.isfinite(dx.float()).all())
    z = x[7].double() @ W.double().t() + b.double()
    d = (torch.softmax(z, 0) @ W.double() - W[123].double()) * gl[7].double()
    check("dx", host(dx[7]), d.cpu().numpy(), dtype, BAR[dtype])
    ok = [i for i in range(300) if t[i] != 123]
    check("loss", host(loss[ok]), host(want[0][ok]), "f32", LOSS)


def test_chunks_of_rows():
    """More exponentials than a chunk holds, the rows that count ending within either chunk."""
    for ignored in (0.0, 0.5):
        t = cuda(*inputs(5000, 16, 128001, "bf16", True, ignored, "mean", 101))
        compare(run(*t), t, "mean", "bf16")


@pytest.mark.parametrize("tile", ["256x256", "128x128"])
def test_tiles(tile, monkeypatch):
    monkeypatch.setenv("MEMSAVE_FUSED_TILE", tile)
    t = cuda(*inputs(515, 264, 20010, "bf16", ignored=0.3, seed=111))
    compare(run(*t), t, "mean", "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(dtype):
    x, W, b, t, gl = inputs(300, 264, 30000, dtype, seed=121)
    want = run(*cuda(x, W, b, t, gl))
    xt, Wt = x.t().contiguous().cuda().t(), W.t().contiguous().cuda().t()
    off = torch.empty(300 * 264 + 1, dtype=x.dtype, device="cuda")[1:].view(300, 264)
    off.copy_(x)
    Wo = torch.empty(30000 * 264 + 1, dtype=x.dtype, device="cuda")[1:].view(30000, 264)
    Wo.copy_(W)
    bo = torch.empty(30001, dtype=x.dtype, device="cuda")[1:]
    bo.copy_(b)
    for a, w, c in ((xt, Wt, b.cuda()), (off, W.cuda(), b.cuda()), (off, Wo, bo)):
        loss, dx = run(a, w, c, *cuda(t, gl))
        if dtype == "f32" and w is Wo:   # 4-byte loads, in another order of the sums
            check("loss", host(loss), host(want[0]), dtype, LOSS)
            check("dx", host(dx), host(want[1]), dtype, BAR[dtype])
            continue
        assert torch.equal(loss, want[0]) and torch.equal(dx, want[1])


def test_account_and_inputs_changed_in_between():
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, "bf16", seed=131))
    want = run(x, W, b, t, gl)
    live = ms.ledger_read()[0]
    m = msa.MSLinearCrossEntropy(W, b)
    m.weight.requires_grad_(False)
    m.bias.requires_grad_(False)
    xg = x.clone().requires_grad_()
    loss = m(xg, t)
    assert ms.ledger_read()[0] - live == 300 * 264 * 3
    with torch.no_grad():   # nothing of these is needed any more
        xg.zero_()
        t.zero_()
        m.weight.zero_()
    loss.backward(gl[0])
    assert ms.ledger_read()[0] == live
    assert torch.equal(xg.grad, want[1]) and torch.equal(loss.reshape(1), want[0])


def test_a_bias_that_trains_keeps_x():
    x, W, b, t, gl = cuda(*inputs(300, 264, 30000, "bf16", seed=141))
    for mask in (2, 3, 4, 5, 7):
        _, rec = ms.layer_forward(ms.LinearCrossEntropy(t), x, W, b, mask)
        assert "grad" not in rec.saved and "x" in rec.saved
        rec.free()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_another_stream_and_a_graph(dtype):
    args = cuda(*inputs(300, 264, 30000, dtype, ignored=0.2, seed=151))
    want = run(*args)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        other = run(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = run(*args)
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = run(*args)
        for a, c, d, e in zip(want, other, got, again):
            assert torch.equal(a, c) and torch.equal(a, d) and torch.equal(a, e)


def test_gradient_against_differences():
    x, W, b, t, gl = cuda(*inputs(64, 130, 260000, "f32", seed=161))
    _, dx = run(x, W, b, t, gl, "sum")
    g = torch.Generator(device="cuda").manual_seed(1)
    d = torch.randn(x.shape, generator=g, device="cuda")
    h = 1e-2
    up, down = (reference(x.double() + s * h * d.double(), W, b, t, gl, "sum")[0] for s in (1, -1))
    got, want = (dx.double() * d.double()).sum().item(), ((up - down) / (2 * h) * gl.double()).item()
    # the central difference's own error: h^2 / 6 times a third derivative of the size of the sum itself
    assert abs(got - want) <= 1e-3 * (dx.double() * d.double()).norm().item()
