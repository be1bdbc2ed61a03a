"""Cross entropy of a linear head against the formulas in 64 bits.

Bars (normwise, max |got - ref| / max |ref|), from the arithmetic.  The loss:
logits are fp32 sums of exact products, their errors below 2^-24 times the root
of D times the logits' size (some 10), and so are lse's: 2e-5 of the largest
loss has an order of room.  Gradients in fp32: the same errors in exp(z - lse),
then sums of at most some 1e4 terms: 5e-5.  In bf16: dz is rounded once (2^-9 a
term, averaging out), the result once more (2^-9): 2^-7 is twice their sum.
"""
import numpy as np
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import TORCH_DT, check, guarded_empty, guards_intact, host

pytestmark = pytest.mark.gpu

LOSS = 2e-5
BAR = {"f32": 5e-5, "bf16": 2.0 ** -7}
IGNORE = -100


def ref(x, W, b, t, g, reduction, ignore=IGNORE):
    """(loss, dx, dW, db) over the rows that count; g is the loss's gradient."""
    live = np.flatnonzero(t != ignore)
    xl, tl = x[live], t[live]
    z = xl @ W.T + (0.0 if b is None else b)
    top = z.max(1, keepdims=True)
    lse = top[:, 0] + np.log(np.exp(z - top).sum(1))
    each = np.zeros(len(t))
    each[live] = lse - z[np.arange(len(live)), tl]
    n = len(live)
    w = g[live] if reduction == "none" else np.full(n, g[0] / (n if reduction == "mean" and n else 1))
    dz = np.exp(z - lse[:, None])
    dz[np.arange(n), tl] -= 1.0
    dz *= w[:, None]
    dx = np.zeros_like(x)
    dx[live] = dz @ W
    loss = each if reduction == "none" else np.array([each.sum() / (n if reduction == "mean" else 1)])
    return loss, dx, dz.T @ xl, dz.sum(0)


def draw(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TORCH_DT[dtype])


def inputs(M, D, V, dtype, bias=True, ignored=0.0, reduction="mean", seed=0):
    g = torch.Generator().manual_seed(seed + 9)
    t = torch.randint(0, V, (M,), generator=g)
    t[torch.rand(M, generator=g) < ignored] = IGNORE
    if M > 1 and reduction == "mean":
        t[M // 2] = V - 1
    gl = torch.rand(M if reduction == "none" else 1, generator=g) + 0.5
    return (draw((M, D), dtype, seed), draw((V, D), dtype, seed + 1, 3.0 * D ** -0.5),
            draw(V, dtype, seed + 2) if bias else None, t, gl)


def run(x, W, b, t, gl, reduction, mask, ignore=IGNORE):
    loss, rec = ms.layer_forward(ms.LinearCrossEntropy(t, ignore, reduction), x, W, b, mask)
    return (loss,) + (ms.layer_backward(rec, gl) if mask else (None,) * 3)


def cuda(*ts):
    return tuple(None if v is None else v.cuda() for v in ts)


def compare(outs, t, reduction, mask, dtype, ignore=IGNORE):
    x, W, b, tgt, gl = t
    refs = ref(x.double().numpy(), W.double().numpy(), None if b is None else b.double().numpy(), tgt.numpy(), gl.double().numpy(),
               reduction, ignore)
    check("loss", host(outs[0]), refs[0], "f32", LOSS)
    for bit, o, r, name in ((1, outs[1], refs[1], "dx"), (2, outs[2], refs[2], "dW"), (4, outs[3], refs[3], "db")):
        assert (o is not None) == bool(mask & bit)
        if o is not None:
            check(name, host(o), r, dtype, BAR[dtype])


# single rows, a few, ragged rows, widths and vocabularies, whole tiles and past them
SHAPES = [(1, 1, 2), (1, 64, 1000), (2, 72, 257), (4, 513, 999), (16, 96, 2050), (17, 40, 300), (100, 130, 259), (129, 64, 128),
          (255, 200, 1025), (256, 128, 256), (300, 96, 513), (1030, 48, 1000), (70, 24, 9001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    t = inputs(*shape, dtype)
    compare(run(*cuda(*t), "mean", 7), t, "mean", 7, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_word(dtype):
    """A vocabulary of one word: no loss and no gradient."""
    t = inputs(5, 16, 1, dtype, reduction="none")
    outs = run(*cuda(*t), "none", 7)
    assert all(float(o.abs().max()) < 1e-5 for o in outs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("ignored", [0.0, 0.4, 0.95])
def test_reductions_and_ignored_rows(ignored, reduction, dtype):
    t = inputs(330, 88, 700, dtype, True, ignored, reduction, 11)
    outs = run(*cuda(*t), reduction, 7)
    compare(outs, t, reduction, 7, dtype)
    dead = (t[3] == IGNORE).cuda()
    assert not outs[1][dead].any()
    if reduction == "none":
        assert not outs[0][dead].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("mask", range(8))
def test_masks(mask, bias, dtype):
    if mask & 4 and not bias:
        pytest.skip("no bias to differentiate")
    t = inputs(150, 72, 520, dtype, bias, 0.2, "sum", 21)
    compare(run(*cuda(*t), "sum", mask), t, "sum", mask, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(40, 64, 1025), (300, 96, 513), (300, 515, 130), (70, 515, 2049), (1030, 203, 777)])
def test_gradients_stay_in_their_rows(shape, dtype):
    """Words that are no multiple of 4 and widths that are none of 8: W's gradient is
    written in place, and nothing past it."""
    M, D, V = shape
    t = inputs(*shape, dtype, ignored=0.2, seed=241)
    x, W, b, tgt, gl = cuda(*t)
    _, rec = ms.layer_forward(ms.LinearCrossEntropy(tgt), x, W, b, 7)
    outs = [guarded_empty(s, dtype) for s in ((M, D), (V, D), (V,))]
    ms.layer_backward(rec, gl, *(o[0] for o in outs))
    torch.cuda.synchronize()
    refs = ref(*(v.double().numpy() for v in t[:3]), t[3].numpy(), t[4].double().numpy(), "mean")[1:]
    for o, r, name in zip(outs, refs, ("dx", "dW", "db")):
        check(name, host(o[0]), r, dtype, BAR[dtype])
        assert guards_intact(o[1], o[2])


@pytest.mark.parametrize("mask", [4, 7])
@pytest.mark.parametrize("shape", [(300, 64, 130), (1030, 264, 2050), (2000, 64, 10007)])
def test_bias_gradient_rounds_once(shape, mask):
    """bf16: the sums of dz from before its rounding, so no more than the result's own
    (at most 2^-8 of a value, and fp32's errors), whatever the factor that every row shares."""
    for factor in (0.7, 1.1):
        t = inputs(*shape, "bf16", ignored=0.1, reduction="sum", seed=231)[:4] + (torch.tensor([factor]),)
        got = run(*cuda(*t), "sum", mask)[3]
        want = ref(*(v.double().numpy() for v in t[:3]), t[3].numpy(), t[4].double().numpy(), "sum")[3]
        err = np.abs(host(got) - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + 2e-5 * np.abs(want).max()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_every_row_ignored(reduction, dtype):
    x, W, b, t, gl = inputs(40, 32, 100, dtype, reduction=reduction)
    t[:] = IGNORE
    loss, dx, dW, db = run(*cuda(x, W, b, t, gl), reduction, 7)
    assert torch.isnan(loss).all() if reduction == "mean" else not loss.any()
    assert not dx.any() and not dW.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_no_rows(reduction, dtype):
    x, W, b, t, gl = inputs(0, 32, 100, dtype, reduction=reduction)
    loss, dx, dW, db = run(*cuda(x, W, b, t, gl), reduction, 7)
    assert loss.shape == ((0,) if reduction == "none" else (1,)) and dx.shape == (0, 32)
    if reduction != "none":
        assert torch.isnan(loss).all() if reduction == "mean" else not loss.any()
    assert not dW.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_whatever_an_ignored_row_holds(bad, dtype):
    t = inputs(90, 64, 300, dtype, True, 0.3, "mean", 31)
    clean = run(*cuda(*t), "mean", 7)
    x = t[0].clone()
    x[t[3] == IGNORE] = bad
    dirty = run(*cuda(x, *t[1:]), "mean", 7)
    assert all(torch.equal(p, q) for p, q in zip(clean, dirty))


def test_a_bad_row_stays_in_its_row():
    x, W, b, t, gl = inputs(60, 64, 300, "bf16", reduction="none", seed=41)
    x[7, 3] = float("nan")
    loss, dx, _, _ = run(*cuda(x, W, b, t, gl), "none", 1)
    rest = [i for i in range(60) if i != 7]
    r = ref(x[rest].double().numpy(), W.double().numpy(), b.double().numpy(), t[rest].numpy(), gl[rest].double().numpy(), "none")
    check("loss", host(loss)[rest], r[0], "f32", LOSS)
    check("dx", host(dx)[rest], r[1], "bf16", BAR["bf16"])
    assert torch.isnan(loss[7]) and torch.isnan(dx[7]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [float("-inf"), -3.0e38])
def test_masked_words(low, dtype):
    """Words that the bias rules out, whole tiles of them: no probability, no
    gradient, and no NaN from a tile that holds no other word."""
    x, W, b, t, gl = inputs(50, 64, 900, dtype, reduction="sum", seed=51)
    b[256:700] = low
    t = torch.where((t >= 256) & (t < 700), 3, t)
    outs = run(*cuda(x, W, b, t, gl), "sum", 7)
    out = torch.arange(256, 700)
    keep = np.r_[0:256, 700:900]
    r = ref(x.double().numpy(), W[keep].double().numpy(), b[keep].double().numpy(),
            np.where(t.numpy() >= 700, t.numpy() - 444, t.numpy()), gl.double().numpy(), "sum")
    check("loss", host(outs[0]), r[0], "f32", LOSS)
    check("dx", host(outs[1]), r[1], dtype, BAR[dtype])
    check("dW", host(outs[2])[keep], r[2], dtype, BAR[dtype])
    assert not outs[2][out.cuda()].any() and not outs[3][out.cuda()].any()


def test_a_masked_target_costs_infinity():
    x, W, b, t, gl = inputs(4, 16, 50, "bf16", reduction="none")
    b[5] = float("-inf")
    t[2] = 5
    loss, dx, _, _ = run(*cuda(x, W, b, t, gl), "none", 1)
    assert torch.isposinf(loss[2]) and torch.isfinite(loss[[0, 1, 3]]).all() and torch.isfinite(dx).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("word", [50, -1, 2 ** 40])
def test_targets_that_are_no_word(word, dtype):
    x, W, b, t, gl = inputs(6, 16, 50, dtype, reduction="none")
    t[3] = word
    loss, dx, _, _ = run(*cuda(x, W, b, t, gl), "none", 1)
    rest = [0, 1, 2, 4, 5]
    assert torch.isnan(loss[3]) and torch.isfinite(loss[rest]).all()
    assert torch.isnan(dx[3]).all() and torch.isfinite(dx[rest]).all()


def test_another_ignored_index():
    t = list(inputs(64, 32, 200, "bf16", reduction="sum"))
    t[3] = torch.where(torch.arange(64) % 3 == 0, 7, t[3])   # a word of the vocabulary that does not count
    compare(run(*cuda(*t), "sum", 7, ignore=7), t, "sum", 7, "bf16", ignore=7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits in the hundreds: the largest carries the sum."""
    x, W, b, t, gl = inputs(33, 64, 400, dtype, reduction="none", seed=61)
    t_ = (x * 40, W, b, t, gl)
    compare(run(*cuda(*t_), "none", 7), t_, "none", 7, dtype)


def test_pieces_of_the_vocabulary():
    """More dz than one piece holds: pieces add up in dx and meet in dW."""
    M, D, V = 6000, 40, 100003
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(M, D, device="cuda", generator=g).bfloat16()
    W = (torch.randn(V, D, device="cuda", generator=g) * 0.3).bfloat16()
    b = torch.randn(V, device="cuda", generator=g).bfloat16()
    t = torch.randint(0, V, (M,), device="cuda", generator=g)
    t[::3] = IGNORE
    one = torch.ones(1, device="cuda")
    loss, dx, dW, db = run(x, W, b, t, one, "mean", 7)
    live = t != IGNORE
    n = int(live.sum())
    want, gx, gW, gb = 0.0, torch.zeros(M, D, device="cuda", dtype=torch.float64), 0.0, 0.0
    for i in range(0, M, 1000):
        rows = torch.arange(i, i + 1000, device="cuda")[live[i:i + 1000]]
        xi, ti = x[rows].double(), t[rows]
        z = xi @ W.double().t() + b.double()
        lse = torch.logsumexp(z, 1)
        want += float((lse - z[torch.arange(len(ti)), ti]).sum()) / n
        dz = torch.exp(z - lse[:, None])
        dz[torch.arange(len(ti)), ti] -= 1.0
        dz /= n
        gx[rows] = dz @ W.double()
        gW, gb = gW + dz.t() @ xi, gb + dz.sum(0)
    check("loss", host(loss), np.array([want]), "f32", LOSS)
    for name, o, r in (("dx", dx, gx), ("dW", dW, gW), ("db", db, gb)):
        check(name, host(o), r.cpu().numpy(), "bf16", BAR["bf16"])


def test_records():
    x, W, b, t, gl = cuda(*inputs(32, 48, 64, "bf16"))
    for mask in range(1, 8):
        live = ms.ledger_read()[0]
        _, rec = ms.layer_forward(ms.LinearCrossEntropy(t), x, W, b, mask)
        a = rec.account()
        assert a["saved_activation_bytes"] == 32 * 48 * 2 + 32 * 12
        assert a["referenced_param_bytes"] == (64 * 48 + 64) * 2
        assert set(rec.saved) == {"x", "W", "b", "lse", "target"}
        assert ms.ledger_read()[0] - live == a["saved_activation_bytes"]
        ms.layer_backward(rec, gl)
        assert ms.ledger_read()[0] == live


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 50])
def test_strides(D, dtype):
    """Transposed and sliced operands, gradients inside larger tensors."""
    M, V = 40, 156
    x, W, b, t, gl = inputs(M, 2 * D, V, dtype, seed=71)
    x, W = x[:, ::2], W[:, ::2]
    xc, Wc = x.t().contiguous().t().cuda(), W.t().contiguous().t().cuda()
    _, rec = ms.layer_forward(ms.LinearCrossEntropy(t.cuda()), xc, Wc, b.cuda(), 7)
    loss, _ = ms.layer_forward(ms.LinearCrossEntropy(t.repeat_interleave(2).cuda()[::2]), xc, Wc, b.cuda(), 0)
    gx = torch.zeros(D, M, dtype=x.dtype, device="cuda").t()
    big = torch.zeros(V, 2 * D, dtype=x.dtype, device="cuda")
    out = ms.layer_backward(rec, gl.cuda(), gx, big[:, D:])
    compare((loss,) + out, (x, W, b, t, gl), "mean", 7, dtype)
    assert not big[:, :D].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 2])
def test_any_alignment(off, dtype):
    M, D, V = 37, 64, 301
    t = inputs(M, D, V, dtype, seed=81)
    place = lambda v: torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")[off:off + v.numel()].view(v.shape).copy_(v)
    x, W, b = (place(v) for v in t[:3])
    gx, xbuf, guard = guarded_empty((M, D), dtype)
    gW, wbuf, _ = guarded_empty((V, D), dtype)
    gb, bbuf, _ = guarded_empty((V,), dtype)
    loss, rec = ms.layer_forward(ms.LinearCrossEntropy(t[3].cuda()), x, W, b, 7)
    out = ms.layer_backward(rec, t[4].cuda(), gx, gW, gb)
    compare((loss,) + out, t, "mean", 7, dtype)
    assert all(guards_intact(v, guard) for v in (xbuf, wbuf, bbuf))


def test_gradients_against_differences():
    """Central differences of the loss along a random direction, the forward in 64
    bits at step 1e-5."""
    x, W, b, t, gl = inputs(6, 20, 30, "f32", reduction="none", seed=91)
    p = [v.double().numpy() for v in (x, W, b)]
    f = lambda p: float((ref(p[0], p[1], p[2], t.numpy(), gl.double().numpy(), "none")[0] * gl.double().numpy()).sum())
    grads = run(*cuda(x, W, b, t, gl), "none", 7)[1:]
    rng = np.random.default_rng(3)
    for i, grad in enumerate(grads):
        v = rng.standard_normal(p[i].shape)
        lo, hi = list(p), list(p)
        lo[i], hi[i] = p[i] - 1e-5 * v, p[i] + 1e-5 * v
        d = (f(hi) - f(lo)) / 2e-5
        assert abs(d - float((host(grad) * v).sum())) <= 1e-4 * max(1.0, abs(d))


@pytest.mark.parametrize("M", [4, 500])
def test_repeats_bit_for_bit_and_on_another_stream(M):
    t = cuda(*inputs(M, 256, 3000, "bf16", True, 0.3, "mean", 101))
    first = run(*t, "mean", 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = run(*t, "mean", 7)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))


def test_prepared_calls():
    x, W, b, t, gl = cuda(*inputs(20, 96, 140, "bf16", seed=111))
    want = run(x, W, b, t, gl, "mean", 7)
    gx, gW, gb = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    p = ms.PreparedLayer(ms.LinearCrossEntropy(t), x, W, b, 7, grad_y=gl, grad_x=gx, grad_W=gW, grad_b=gb)
    for _ in range(3):
        p.forward()
        p.backward()
    assert all(torch.equal(o, w) for o, w in zip((p.y, gx, gW, gb), want))


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("mask", [0, 1, 3, 7])
def test_module(mask, reduction):
    t = inputs(24, 72, 140, "f32", True, 0.2, reduction, 121)
    x, W, b, tgt, _ = cuda(*t)
    m = msa.MSLinearCrossEntropy(W, b, reduction=reduction)
    m.weight.requires_grad_(bool(mask & 2))
    m.bias.requires_grad_(bool(mask & 4))
    xc = x.reshape(2, 12, 72).requires_grad_(bool(mask & 1))
    loss = m(xc, tgt.reshape(2, 12))
    assert loss.shape == ((2, 12) if reduction == "none" else ())
    if mask:
        loss.sum().backward()
    t = t[:4] + (torch.ones(24 if reduction == "none" else 1),)
    compare((loss.reshape(-1), xc.grad.reshape(24, 72) if mask & 1 else None, m.weight.grad, m.bias.grad), t, reduction, mask, "f32")


def test_a_changed_target_is_noticed():
    x, W, b, tgt, _ = cuda(*inputs(8, 16, 20, "f32"))
    m = msa.MSLinearCrossEntropy(W, b)
    loss = m(x, tgt)
    tgt.add_(0)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_refusals():
    x, W, b, t, gl = cuda(*inputs(4, 10, 30, "f32"))
    spec = ms.LinearCrossEntropy(t)

    def refused(status, fn):
        with pytest.raises(ms.MemsaveError) as e:
            fn()
        assert e.value.status == status

    refused(3, lambda: ms.layer_forward(spec, x, W[:, :9], b))
    refused(3, lambda: ms.layer_forward(spec, x, W, b[:29].contiguous()))
    refused(4, lambda: ms.layer_forward(spec, x, W.bfloat16(), b))
    refused(4, lambda: ms.layer_forward(spec, x, W, b, y=torch.empty(1, device="cuda", dtype=torch.bfloat16)))
    refused(3, lambda: ms.layer_forward(spec, x, W, b, y=torch.empty(4, device="cuda")))
    refused(2, lambda: ms.layer_forward(spec, x, W, None, 4))
    refused(2, lambda: ms.layer_forward(spec, x, W, b, 16))
    with pytest.raises(ValueError):
        ms.layer_forward(ms.LinearCrossEntropy(t[:3]), x, W, b)
    with pytest.raises(TypeError):
        ms.layer_forward(ms.LinearCrossEntropy(t.int()), x, W, b)
    with pytest.raises(TypeError):
        ms.layer_forward(ms.LinearCrossEntropy(t.cpu()), x, W, b)
    with pytest.raises(ValueError):
        ms.layer_forward(ms.LinearCrossEntropy(t, reduction="max"), x, W, b)
    with pytest.raises(TypeError):
        ms.layer_forward(spec, x, None)
    _, rec = ms.layer_forward(spec, x, W, b, 1)
    refused(4, lambda: ms.layer_backward(rec, gl.bfloat16()))
    refused(3, lambda: ms.layer_backward(rec, torch.ones(4, device="cuda")))
    ms.layer_backward(rec, gl)
    refused(7, lambda: ms.layer_backward(rec, gl, torch.empty_like(x)))
    assert ms.ledger_read()[0] == 0
