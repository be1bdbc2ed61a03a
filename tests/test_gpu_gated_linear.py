"""Gated linear unit forward and backward against the formulas in 64 bits.

Bars (normwise, max |got - ref| / max |ref|), from the arithmetic.  fp32: sums
of D or M products in chains whose errors grow like the root of their length:
below 1e-5 here; 5e-5.  bf16: y is one rounding (2^-9) of an fp32 value; dz is
rounded once before the gradients' products (2^-9 of each term, which average
out; a kept z has 2^-17 and does not count) and the results once more: 2^-7 is
more than twice their sum.
"""
import numpy as np
import pytest
import torch
from scipy import special

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import TORCH_DT, check, guarded_empty, guards_intact, host

pytestmark = pytest.mark.gpu

BAR = {"f32": 5e-5, "bf16": 2.0 ** -7}
ACTS = ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"]


def act64(name, z):
    s = special.expit(z)
    if name == "sigmoid":
        return s, s * special.expit(-z)
    if name == "silu":
        return z * s, s + z * s * special.expit(-z)
    if name == "relu":
        return np.maximum(z, 0), (z > 0).astype(np.float64)
    if name == "gelu":
        c = special.ndtr(z)
        return z * c, c + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    k = np.sqrt(2 / np.pi)
    t = np.tanh(k * (z + 0.044715 * z ** 3))
    return z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t * t) / 2 * k * (1 + 0.134145 * z * z)


def ref(x, W, b, dy, act):
    z = x @ W.T + (0.0 if b is None else b)
    F = W.shape[0] // 2
    a, da = act64(act, z[:, :F])
    u = z[:, F:]
    dz = np.concatenate([dy * u * da, dy * a], 1)
    return a * u, dz @ W, dz.T @ x, dz.sum(0)


def draw(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TORCH_DT[dtype])


def inputs(M, D, F, dtype, bias=True, seed=0):
    return (draw((M, D), dtype, seed), draw((2 * F, D), dtype, seed + 1, D ** -0.5),
            draw(2 * F, dtype, seed + 2, 0.5) if bias else None, draw((M, F), dtype, seed + 3))


def run(x, W, b, dy, act, keep, mask):
    y, rec = ms.layer_forward(ms.GatedLinear(act, keep), x, W, b, mask)
    return (y,) + (ms.layer_backward(rec, dy) if mask else (None,) * 3)


def cuda(*ts):
    return tuple(None if t is None else t.cuda() for t in ts)


def compare(outs, t, act, mask, dtype):
    refs = ref(*(None if v is None else v.double().numpy() for v in t), act)
    check("y", host(outs[0]), refs[0], dtype, BAR[dtype])
    for bit, o, r, name in ((1, outs[1], refs[1], "dx"), (2, outs[2], refs[2], "dW"), (4, outs[3], refs[3], "db")):
        assert (o is not None) == bool(mask & bit)
        if o is not None:
            check(name, host(o), r, dtype, BAR[dtype])


# single tokens, a few, ragged rows and widths, whole tiles and one past them
SHAPES = [(1, 1, 1), (1, 64, 96), (1, 777, 130), (2, 512, 1000), (5, 40, 3), (16, 256, 264), (17, 96, 33), (100, 200, 300),
          (129, 65, 127), (256, 128, 128), (257, 136, 129), (300, 1030, 70), (515, 64, 258), (1025, 72, 520)]


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype, keep):
    t = inputs(*shape, dtype)
    compare(run(*cuda(*t), "silu", keep, 7), t, "silu", 7, dtype)


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype, keep):
    t = inputs(70, 96, 136, dtype, seed=11)
    t = (t[0] * 3, t[1], t[2], t[3])   # projections to 10 and beyond: both tails
    compare(run(*cuda(*t), act, keep, 7), t, act, 7, dtype)


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("mask", range(8))
def test_masks(mask, bias, dtype, keep):
    if mask & 4 and not bias:
        pytest.skip("no bias to differentiate")
    t = inputs(150, 88, 104, dtype, bias, 21)
    compare(run(*cuda(*t), "gelu", keep, mask), t, "gelu", mask, dtype)


@pytest.mark.parametrize("tokens", [1, 3, 8, 15, 16, 31, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_tokens(tokens, dtype):
    t = inputs(tokens, 1160, 1037, dtype, seed=31)
    compare(run(*cuda(*t), "silu", "projections", 0), t, "silu", 0, dtype)


def test_large_tiles():
    """Enough rows and columns for the widest tile."""
    t = inputs(4100, 256, 2060, "bf16", seed=41)
    dev = cuda(*t)
    for keep in ("projections", "input"):
        outs = run(*dev, "silu", keep, 7)
        x, W, b, dy = (v.double().cuda() for v in t)
        z = x @ W.t() + b
        s = torch.sigmoid(z[:, :2060])
        u = z[:, 2060:]
        dz = torch.cat([dy * u * (s + z[:, :2060] * s * (1 - s)), dy * z[:, :2060] * s], 1)
        for name, o, r in zip(("y", "dx", "dW", "db"), outs, (z[:, :2060] * s * u, dz @ W, dz.t() @ x, dz.sum(0))):
            check(name, host(o), r.cpu().numpy(), "bf16", BAR["bf16"])


@pytest.mark.parametrize("keep", ["projections", "input"])
def test_records(keep):
    x, W, b, dy = cuda(*inputs(32, 48, 64, "bf16"))
    for mask in range(1, 8):
        live = ms.ledger_read()[0]
        _, rec = ms.layer_forward(ms.GatedLinear("silu", keep), x, W, b, mask)
        a = rec.account()
        if keep == "input":
            assert a["saved_activation_bytes"] == 32 * 48 * 2
            assert a["referenced_param_bytes"] == (2 * 64 * 48 + 2 * 64) * 2
            assert set(rec.saved) == {"x", "W", "b"}
        else:
            assert a["saved_activation_bytes"] == 32 * 128 * 3 + (32 * 48 * 2 if mask & 2 else 0)
            assert a["referenced_param_bytes"] == (2 * 64 * 48 * 2 if mask & 1 else 0)
            assert set(rec.saved) == {"projections"} | ({"x"} if mask & 2 else set()) | ({"W"} if mask & 1 else set())
        assert ms.ledger_read()[0] - live == a["saved_activation_bytes"]
        ms.layer_backward(rec, dy)
        assert ms.ledger_read()[0] == live


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype, keep):
    x, W, b, dy = cuda(*inputs(0, 24, 16, dtype))
    y, dx, dW, db = run(x, W, b, dy, "silu", keep, 7)
    assert y.shape == (0, 16) and dx.shape == (0, 24)
    assert not dW.any() and not db.any()


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 50])
def test_strides(D, dtype, keep):
    """Transposed, sliced and broadcast operands, outputs inside larger tensors."""
    M, F = 40, 56
    x, W, b, dy = inputs(M, 2 * D, F, dtype, seed=51)
    x, W, dy = x[:, ::2], W[:, ::2], dy[:1].expand(M, F)
    W = W * 2 ** 0.5
    xc, Wc = x.t().contiguous().t().cuda(), W.t().contiguous().t().cuda()
    big = torch.zeros(M, 2 * F, dtype=x.dtype, device="cuda")
    y, rec = ms.layer_forward(ms.GatedLinear("silu", keep), xc, Wc, b.cuda(), 7, y=big[:, F:])
    gx = torch.zeros(D, M, dtype=x.dtype, device="cuda").t()
    gW = torch.zeros(2 * F, 2 * D, dtype=x.dtype, device="cuda")[:, ::2]
    out = ms.layer_backward(rec, dy[:1].cuda().expand(M, F), gx, gW)
    compare((y,) + out, (x, W, b, dy), "silu", 7, dtype)
    assert not big[:, :F].any()


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 2])
def test_any_alignment(off, dtype, keep):
    M, D, F = 37, 64, 41
    t = inputs(M, D, F, dtype, seed=61)
    place = lambda v: torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")[off:off + v.numel()].view(v.shape).copy_(v)
    x, W, b, dy = (place(v) for v in t)
    y, ybuf, guard = guarded_empty((M, F), dtype)
    gx, xbuf, _ = guarded_empty((M, D), dtype)
    gW, wbuf, _ = guarded_empty((2 * F, D), dtype)
    _, rec = ms.layer_forward(ms.GatedLinear("gelu", keep), x, W, b, 7, y=y)
    out = ms.layer_backward(rec, dy, gx, gW)
    compare((y,) + out, t, "gelu", 7, dtype)
    assert guards_intact(ybuf, guard) and guards_intact(xbuf, guard) and guards_intact(wbuf, guard)


@pytest.mark.parametrize("keep", ["projections", "input"])
def test_bad_values_stay_in_their_row(keep):
    x, W, b, dy = inputs(20, 64, 48, "bf16", seed=71)
    x[7, 3] = float("nan")
    y, dx, _, _ = run(*cuda(x, W, b, dy), "silu", keep, 1)
    rest = [i for i in range(20) if i != 7]
    r = ref(*(v.double().numpy() for v in (x[rest], W, b, dy[rest])), "silu")
    check("y", host(y)[rest], r[0], "bf16", BAR["bf16"])
    check("dx", host(dx)[rest], r[1], "bf16", BAR["bf16"])
    assert torch.isnan(y[7]).all() and torch.isnan(dx[7]).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_gradients_against_differences(act):
    """Central differences of sum(dy y) along a random direction, the forward in
    64 bits at step 1e-5."""
    t = tuple(v.double().numpy() for v in inputs(6, 20, 9, "f32", seed=81))
    grads = run(*cuda(*(torch.from_numpy(v).float() for v in t)), act, "input", 7)[1:]
    rng = np.random.default_rng(2)
    for i, grad in enumerate(grads):
        v = rng.standard_normal(t[i].shape)
        lo, hi = list(t), list(t)
        lo[i], hi[i] = t[i] - 1e-5 * v, t[i] + 1e-5 * v
        d = float(((ref(*hi, act)[0] - ref(*lo, act)[0]) * t[3]).sum()) / 2e-5
        assert abs(d - float((host(grad) * v).sum())) <= 1e-4 * max(1.0, abs(d))


@pytest.mark.parametrize("M", [4, 300])
def test_repeats_bit_for_bit_and_on_another_stream(M):
    t = cuda(*inputs(M, 256, 320, "bf16", seed=91))
    first = run(*t, "silu", "input", 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = run(*t, "silu", "input", 7)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))


@pytest.mark.parametrize("keep", ["projections", "input"])
def test_prepared_calls(keep):
    x, W, b, dy = cuda(*inputs(20, 96, 40, "bf16", seed=101))
    want = run(x, W, b, dy, "silu", keep, 7)
    gx, gW, gb = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    p = ms.PreparedLayer(ms.GatedLinear("silu", keep), x, W, b, 7, grad_y=dy, grad_x=gx, grad_W=gW, grad_b=gb)
    for _ in range(3):
        p.forward()
        p.backward()
    assert all(torch.equal(o, w) for o, w in zip((p.y, gx, gW, gb), want))


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("mask", [0, 1, 3, 7])
def test_module(mask, keep):
    t = inputs(24, 72, 40, "f32", seed=111)
    x, W, b, dy = cuda(*t)
    m = msa.MSGatedLinear(W, b, "silu", keep)
    m.weight.requires_grad_(bool(mask & 2))
    m.bias.requires_grad_(bool(mask & 4))
    xc = x.reshape(2, 12, 72).requires_grad_(bool(mask & 1))
    y = m(xc)
    if mask:
        y.backward(dy.reshape(y.shape))
    compare((y.reshape(24, 40), xc.grad.reshape(24, 72) if mask & 1 else None, m.weight.grad, m.bias.grad), t, "silu", mask, "f32")


def test_refusals():
    x, W, b, dy = cuda(*inputs(4, 10, 6, "f32"))
    spec = ms.GatedLinear()

    def refused(status, fn):
        with pytest.raises(ms.MemsaveError) as e:
            fn()
        assert e.value.status == status

    refused(3, lambda: ms.layer_forward(spec, x, W[:11], None))
    refused(3, lambda: ms.layer_forward(spec, x, W[:, :9], None))
    refused(3, lambda: ms.layer_forward(spec, x, W, b[:6].contiguous()))
    refused(4, lambda: ms.layer_forward(spec, x, W.bfloat16(), None))
    refused(4, lambda: ms.layer_forward(spec, x, W, b.bfloat16()))
    refused(5, lambda: ms.layer_forward(spec, x, W, b, y=torch.empty(1, 6, device="cuda").expand(4, 6)))
    refused(2, lambda: ms.layer_forward(spec, x, W, None, 4))
    refused(2, lambda: ms.layer_forward(spec, x, W, b, 8))
    with pytest.raises(ValueError):
        ms.layer_forward(ms.GatedLinear("swish2"), x, W, b)
    with pytest.raises(ValueError):
        ms.layer_forward(ms.GatedLinear(keep="nothing"), x, W, b)
    with pytest.raises(TypeError):
        ms.layer_forward(spec, x, None)
    with pytest.raises(TypeError):
        ms.layer_forward(spec, x.cpu(), W, b)
    with pytest.raises(ValueError):
        ms.layer_forward(spec, x.reshape(2, 2, 10), W, b)
    _, rec = ms.layer_forward(spec, x, W, b, 1)
    refused(3, lambda: ms.layer_backward(rec, dy[:, :5]))
    ms.layer_backward(rec, dy)
    refused(7, lambda: ms.layer_backward(rec, dy, torch.empty_like(x)))
    assert ms.ledger_read()[0] == 0
