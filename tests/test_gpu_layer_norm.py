"""Layer norm forward and backward against the formulas in 64 bits.

Bars (normwise, max |got - ref| / max |ref|), from the arithmetic: bf16
results are one rounding of a 32-bit value, half a unit in 2^8, so 2^-8 has
twice the room; 32-bit results come from sums of at most some 2^14 terms taken
in 64 or more chains (rounding errors below sqrt(2^14 / 64) * 2^-24 * a few),
so 2e-5 has two orders of room.  dx is a difference of terms as
large as r |q| (q = dy gamma, r = 1 / sqrt(var + eps)), which cancel where a row
has few elements (of two, all but some eps r^2): its error is measured against
the larger of dx and those terms.
"""
import numpy as np
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import TORCH_DT, check, guarded_empty, guards_intact, host

pytestmark = pytest.mark.gpu

BAR = {"f32": 2e-5, "bf16": 2.0 ** -8}
EPS = 1e-5


def ref(x, g, b, dy, eps=EPS):
    D = x.shape[1]
    g = np.ones(D) if g is None else g
    c = x - x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    h = c * r
    q = dy * g
    dx = r * (q - q.mean(1, keepdims=True) - h * (q * h).mean(1, keepdims=True))
    return h * g + (0.0 if b is None else b), dx, (dy * h).sum(0), dy.sum(0), np.abs(r * q).max(initial=0.0)


def draw(shape, dtype, seed, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(TORCH_DT[dtype])


def inputs(M, D, dtype, seed=0):
    return (draw((M, D), dtype, seed, 1.5, 0.7), draw(D, dtype, seed + 1, 0.3, 1.0), draw(D, dtype, seed + 2, 0.5),
            draw((M, D), dtype, seed + 3))


def run(x, g, b, dy, mask):
    y, rec = ms.layer_forward(ms.LayerNorm(EPS), x, g, b, mask)
    return (y,) + (ms.layer_backward(rec, dy) if mask else (None,) * 3)


def check_dx(got, dx, terms, dtype):
    """Normwise, the terms' size taking part in the norm."""
    check("dx", np.append(got.ravel(), terms), np.append(dx.ravel(), terms), dtype, BAR[dtype])


def compare(outs, refs, mask, dtype):
    check("y", host(outs[0]), refs[0], dtype, BAR[dtype])
    for bit, o, r, name in ((1, outs[1], refs[1], "dx"), (2, outs[2], refs[2], "dgamma"), (4, outs[3], refs[3], "dbeta")):
        assert (o is not None) == bool(mask & bit)
        if o is None:
            continue
        if bit == 1:
            check_dx(host(o), r, refs[4], dtype)
        else:
            check(name, host(o), r, dtype, BAR[dtype])


# one element to past the registers; widths that no vector divides
SHAPES = [(1, 2), (1, 768), (3, 5), (7, 64), (33, 257), (130, 515), (5, 2048), (4, 2049), (9, 4096), (3, 8192), (2, 8193),
          (3, 12288), (2, 12291), (5, 6145), (2100, 66), (4097, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    x, g, b, dy = inputs(*shape, dtype)
    outs = run(x.cuda(), g.cuda(), b.cuda(), dy.cuda(), 7)
    compare(outs, ref(*(t.double().numpy() for t in (x, g, b, dy))), 7, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", range(8))
@pytest.mark.parametrize("D", [100, 2304, 12296])
def test_masks(D, mask, dtype):
    x, g, b, dy = inputs(11, D, dtype, 5)
    outs = run(x.cuda(), g.cuda(), b.cuda(), dy.cuda(), mask)
    compare(outs, ref(*(t.double().numpy() for t in (x, g, b, dy))), mask, dtype)


@pytest.mark.parametrize("has_g,has_b,mask", [(False, False, 1), (True, False, 3), (False, True, 5)])
@pytest.mark.parametrize("D", [96, 12290])
def test_without_scale_or_shift(has_g, has_b, mask, D):
    x, g, b, dy = inputs(6, D, "f32", 9)
    g, b = g if has_g else None, b if has_b else None
    outs = run(x.cuda(), g.cuda() if has_g else None, b.cuda() if has_b else None, dy.cuda(), mask)
    compare(outs, ref(*(None if t is None else t.double().numpy() for t in (x, g, b, dy))), mask, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keeps_the_input_alone(dtype):
    x, g, b, dy = (t.cuda() for t in inputs(12, 80, dtype))
    n, e = x.numel() * x.element_size(), x.element_size()
    for mask in range(1, 8):
        live = ms.ledger_read()[0]
        _, rec = ms.layer_forward(ms.LayerNorm(EPS), x, g, b, mask)
        a = rec.account()
        assert a["saved_activation_bytes"] == (n if mask & 3 else 0) == ms.ledger_read()[0] - live
        assert a["referenced_param_bytes"] == (80 * e if mask & 1 else 0)
        assert set(rec.saved) == ({"x"} if mask & 3 else set()) | ({"W"} if mask & 1 else set())
        ms.layer_backward(rec, dy)
        assert ms.ledger_read()[0] == live


def test_no_rows():
    x, g, b, dy = (t.cuda() for t in inputs(0, 70, "f32"))
    y, dx, dg, db = run(x, g, b, dy, 7)
    assert y.shape == dx.shape == (0, 70)
    assert not dg.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 3000])
def test_strides(D, dtype):
    """Sliced, transposed and broadcast operands; outputs inside a larger tensor."""
    x, g, b, dy = inputs(10, 2 * D, dtype, 3)
    x, dy, g, b = x[:, ::2], dy[:1, ::2].expand(10, D), g[:D], b[:D]
    refs = ref(*(t.double().numpy() for t in (x, g, b, dy)))
    xc = x.t().contiguous().t().cuda()
    big = torch.zeros(10, 2 * D, dtype=x.dtype, device="cuda")
    y, rec = ms.layer_forward(ms.LayerNorm(EPS), xc, g.cuda(), b.cuda(), 7, y=big[:, D:])
    gx = torch.zeros(D, 10, dtype=x.dtype, device="cuda").t()
    assert rec.saved["x"] is xc
    out = ms.layer_backward(rec, dy[:1].cuda().expand(10, D), gx)
    compare((y,) + out, refs, 7, dtype)
    assert not big[:, :D].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 3])
def test_any_alignment(off, dtype):
    D, M = 203, 9
    x, g, b, dy = inputs(M, D, dtype, 21)
    place = lambda t: torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")[off:off + t.numel()].view(t.shape).copy_(t)
    y, ybuf, guard = guarded_empty((M, D), dtype)
    gx, xbuf, _ = guarded_empty((M, D), dtype)
    _, rec = ms.layer_forward(ms.LayerNorm(EPS), place(x), place(g), place(b), 7, y=y)
    _, dg, db = ms.layer_backward(rec, place(dy), gx)
    compare((y, gx, dg, db), ref(*(t.double().numpy() for t in (x, g, b, dy))), 7, dtype)
    assert guards_intact(ybuf, guard) and guards_intact(xbuf, guard)


def test_offset_rows_and_constant_rows():
    """A mean far from zero takes nothing from the variance; a constant row has
    no variance and gives the shift."""
    x, g, b, dy = inputs(8, 1000, "f32", 31)
    x += 1000.0
    x[3] = 7.25
    x64 = x.double().numpy()
    y, dx, dg, db = run(x.cuda(), g.cuda(), b.cuda(), dy.cuda(), 7)
    refs = ref(x64, g.double().numpy(), b.double().numpy(), dy.double().numpy())
    rest = [0, 1, 2, 4, 5, 6, 7]
    # the mean is rounded to 2^-24 of 1000, and h moves by that
    check("y", host(y)[rest], refs[0][rest], "f32", 5e-4)
    assert np.array_equal(host(y)[3], b.double().numpy())
    one = ref(x64[3:4], g.double().numpy(), b.double().numpy(), dy[3:4].double().numpy())
    check_dx(host(dx)[3:4], one[1], one[4], "f32")


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_bad_values_stay_in_their_row(bad):
    x, g, b, dy = inputs(9, 300, "f32", 41)
    x[4, 17] = bad
    y, dx, _, db = run(x.cuda(), g.cuda(), b.cuda(), dy.cuda(), 7)
    keep = [i for i in range(9) if i != 4]
    r = ref(x[keep].double().numpy(), g.double().numpy(), b.double().numpy(), dy[keep].double().numpy())
    check("y", host(y)[keep], r[0], "f32", BAR["f32"])
    check_dx(host(dx)[keep], r[1], r[4], "f32")
    assert torch.isnan(y[4]).all() and torch.isnan(dx[4]).all() and torch.isfinite(db).all()


def test_gradients_against_differences():
    """Central differences of sum(dy y) in the direction of a random vector, the
    forward in 64 bits, step 1e-5 (error below 1e-8)."""
    x, g, b, dy = (t.double().numpy() for t in inputs(5, 37, "f32", 51))
    f = lambda x, g, b: float((ref(x, g, b, dy)[0] * dy).sum())
    grads = run(*(torch.from_numpy(t).float().cuda() for t in (x, g, b, dy)), 7)[1:]
    rng = np.random.default_rng(1)
    for i, grad in enumerate(grads):
        v = rng.standard_normal((x, g, b)[i].shape)
        lo, hi = [x, g, b], [x, g, b]
        lo[i], hi[i] = lo[i] - 1e-5 * v, hi[i] + 1e-5 * v
        d = (f(*hi) - f(*lo)) / 2e-5
        assert abs(d - float((host(grad) * v).sum())) <= 1e-4 * max(1.0, abs(d))


def test_repeats_bit_for_bit_and_on_another_stream():
    x, g, b, dy = (t.cuda() for t in inputs(3000, 200, "bf16", 61))
    first = run(x, g, b, dy, 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = run(x, g, b, dy, 7)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))


def test_prepared_calls():
    x, g, b, dy = (t.cuda() for t in inputs(20, 96, "f32", 71))
    want = run(x, g, b, dy, 7)
    gx, gg, gb = torch.empty_like(x), torch.empty_like(g), torch.empty_like(b)
    p = ms.PreparedLayer(ms.LayerNorm(EPS), x, g, b, 7, grad_y=dy, grad_x=gx, grad_W=gg, grad_b=gb)
    for _ in range(3):
        p.forward()
        p.backward()
    assert all(torch.equal(o, w) for o, w in zip((p.y, gx, gg, gb), want))


@pytest.mark.parametrize("mask", [0, 1, 2, 4, 6, 7])
def test_module(mask):
    x, g, b, dy = inputs(24, 72, "f32", 81)
    m = msa.MSLayerNorm(g.cuda(), b.cuda(), EPS)
    m.weight.requires_grad_(bool(mask & 2))
    m.bias.requires_grad_(bool(mask & 4))
    xc = x.cuda().reshape(2, 3, 4, 72).requires_grad_(bool(mask & 1))
    y = m(xc)
    if mask:
        y.backward(dy.cuda().reshape(y.shape))
    grads = (xc.grad.reshape(24, 72) if mask & 1 else None, m.weight.grad, m.bias.grad)
    compare((y.reshape(24, 72),) + grads, ref(*(t.double().numpy() for t in (x, g, b, dy))), mask, "f32")


def test_convert():
    net = torch.nn.Sequential(torch.nn.Linear(16, 24), torch.nn.LayerNorm(24), torch.nn.LayerNorm((3, 24))).cuda()
    msa.convert(net)
    assert isinstance(net[1], torch.nn.LayerNorm)          # asked for by name only
    w = net[1].weight
    msa.convert(net, layer_norm=True)
    assert isinstance(net[1], msa.MSLayerNorm) and net[1].weight is w
    assert isinstance(net[2], torch.nn.LayerNorm)


def test_refusals():
    x, g, b, dy = (t.cuda() for t in inputs(4, 10, "f32"))
    ln = ms.LayerNorm(EPS)

    def refused(status, fn):
        with pytest.raises(ms.MemsaveError) as e:
            fn()
        assert e.value.status == status

    refused(3, lambda: ms.layer_forward(ln, x, g[:9].contiguous(), b))
    refused(3, lambda: ms.layer_forward(ln, x[:, :0], None, None))
    refused(4, lambda: ms.layer_forward(ln, x, g.bfloat16(), b))
    refused(5, lambda: ms.layer_forward(ln, x, torch.ones(20, device="cuda")[::2], b))
    refused(5, lambda: ms.layer_forward(ln, x, g, b, y=torch.empty(1, 10, device="cuda").expand(4, 10)))
    refused(2, lambda: ms.layer_forward(ln, x, None, b, 2))
    refused(2, lambda: ms.layer_forward(ln, x, g, None, 4))
    refused(2, lambda: ms.layer_forward(ln, x, g, b, 8))
    refused(10, lambda: ms.layer_forward(ms.LayerNorm(float("nan")), x, g, b))
    refused(10, lambda: ms.layer_forward(ms.LayerNorm(-1.0), x, g, b))
    with pytest.raises(TypeError):
        ms.layer_forward(ln, x.half(), g.half(), b.half())
    with pytest.raises(TypeError):
        ms.layer_forward(ln, x.cpu(), g, b)
    with pytest.raises(ValueError):
        ms.layer_forward(ln, x.reshape(2, 2, 10), g, b)
    _, rec = ms.layer_forward(ln, x, g, b, 3)
    refused(3, lambda: ms.layer_backward(rec, dy[:3]))
    refused(4, lambda: ms.layer_backward(rec, dy.bfloat16(), torch.empty_like(x), torch.empty_like(g)))
    ms.layer_backward(rec, dy)
    refused(7, lambda: ms.layer_backward(rec, dy, torch.empty_like(x), torch.empty_like(g)))
    assert ms.ledger_read()[0] == 0
