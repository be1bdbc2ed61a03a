"""Head norms with rotation, forward and backward, against the formulas in 64 bits.

Bars are elementwise.  u is half a step of the type (2^-8 in bf16, 2^-24 in fp32), t = 2^-24.
The sum of D squares is off by at most D t of itself, so z by (D / 2 + 6) t; a cosine or
sine, from an angle reduced in 64 bits and rounded once, by 2^-22:
  y    u |y| + ((D / 2 + 8) t + 2^-22) (|z_i| + |z_j|)
  dx   u |dx| + ((2 D + 24) t + 2^-22) r (|q_i| + |q_j| + |x| r^2 mean |q x|)
  dg   u |dg| + ((D + 24) t + 2^-22 + n t) sum over n rows of (|dz_i| + |dz_j|) |x| r
"""
import math

import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import TORCH_DT, guarded_empty, guards_intact
from test_gpu_attention import U, close, draw

pytestmark = pytest.mark.gpu
EPS = 1e-6
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def turned(z, angle, pairs, back=False):
    half = angle.shape[-1]
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    s = -s if back else s
    out = z.clone()
    i = torch.arange(half, device=z.device)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    out[..., a] = z[..., a] * c - z[..., b] * s
    out[..., b] = z[..., b] * c + z[..., a] * s
    return out


def partner(z, half, pairs):
    """|z| of the element and its partner together."""
    out = z.abs().clone()
    i = torch.arange(half, device=z.device)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    both = z[..., a].abs() + z[..., b].abs()
    out[..., a], out[..., b] = both, both
    return out


def reference(x, gq, gk, gy, pos, freq, q_heads, norm, pairs, dtype, eps=EPS):
    D, u, t = x.shape[2], U[dtype], 2.0 ** -24
    x, gy = x.double(), gy.double()
    H = x.shape[1]
    one = torch.ones(D, dtype=torch.float64, device=x.device)
    g = torch.stack([(one if gq is None else gq.double()) if h < q_heads else (one if gk is None else gk.double()) for h in range(H)])
    if not norm:
        g = torch.ones_like(g)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) if norm else torch.ones_like(x[..., :1])
    angle = torch.zeros(x.shape[0], 0, dtype=torch.float64, device=x.device) if freq is None else pos.double()[:, None] * freq.double()[None]
    half = angle.shape[-1]
    z = x * r * g
    y = turned(z, angle, pairs)
    by = u * y.abs() + ((D / 2 + 8) * t + 2.0 ** -22) * partner(z, half, pairs)
    dz = turned(gy, angle, pairs, True)
    q = dz * g
    m = (q * x).mean(-1, keepdim=True)
    dx = r * (q - x * r * r * m) if norm else dz
    wide = partner(gy, half, pairs)
    bx = u * dx.abs() + ((2 * D + 24) * t + 2.0 ** -22) * r * (wide * g.abs() + (x.abs() * r * r * (wide * g.abs() * x.abs()).mean(-1, keepdim=True)))
    e = dz * x * r
    be = wide * x.abs() * r
    outs, bars = [y, dx], [by, bx]
    for part in (slice(0, q_heads), slice(q_heads, H)):
        s = e[:, part].sum((0, 1))
        n = e[:, part].shape[0] * e[:, part].shape[1]
        outs.append(s)
        bars.append(u * s.abs() + ((D + 24 + n) * t + 2.0 ** -22) * be[:, part].sum((0, 1)))
    return outs, bars


def inputs(T, H, D, dtype, seed=0, far=5000):
    x, gy = draw((T, H, D), dtype, seed, 1.5), draw((T, H, D), dtype, seed + 1)
    gq, gk = 1 + draw((D,), dtype, seed + 2, 0.3), 1 + draw((D,), dtype, seed + 3, 0.3)
    gen = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, far, (T,), generator=gen).to(torch.int32).cuda()
    return x, gq, gk, gy, pos


def run(spec, x, gq, gk, gy, mask, y=None):
    y, rec = ms.layer_forward(spec, x, gq, gk, mask, y=y)
    return [y] + list(ms.layer_backward(rec, gy) if mask else (None,) * 3)


def compare(outs, refs, bars, mask=7):
    for i, name in enumerate(("y", "dx", "dgq", "dgk")):
        if i and not mask >> (i - 1) & 1:
            assert outs[i] is None
            continue
        close(name, outs[i], refs[i], bars[i])


def case(T, q_heads, k_heads, D, R, pairs, dtype, mask=7, seed=0, far=5000, norm=True):
    x, gq, gk, gy, pos = inputs(T, q_heads + k_heads, D, dtype, seed, far)
    if not norm:
        gq = gk = None
    freq = ms.rotary_frequencies(R, device="cuda") if R else None
    refs, bars = reference(x, gq, gk, gy, pos, freq, q_heads, norm, pairs, dtype)
    spec = ms.HeadNormRotary(pos if R else None, freq, q_heads, norm, EPS, pairs)
    compare(run(spec, x, gq, gk, gy, mask), refs, bars, mask)


PAIRS = pytest.mark.parametrize("pairs", [False, True])


@DTYPES
@PAIRS
@pytest.mark.parametrize("D,R", [(1, 0), (2, 2), (3, 2), (8, 8), (16, 16), (20, 12), (32, 32), (33, 30), (40, 40), (64, 64), (64, 32), (72, 48), (80, 80), (90, 36),
                                 (100, 100), (127, 126), (128, 128), (128, 64), (129, 16), (200, 200), (255, 254), (256, 256), (256, 2), (64, 0)])
def test_head_sizes(D, R, pairs, dtype):
    case(37, 3, 2, D, R, pairs, dtype, seed=D + R)


@DTYPES
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 300, 2500])
@pytest.mark.parametrize("heads", [(1, 0), (0, 1), (5, 3), (32, 8)])
def test_rows_and_heads(heads, T, dtype):
    case(T, *heads, 64, 64, False, dtype, seed=T)


@DTYPES
@PAIRS
@pytest.mark.parametrize("mask", range(8))
@pytest.mark.parametrize("D", [64, 100])
def test_masks(D, mask, pairs, dtype):
    case(50, 4, 2, D, D, pairs, dtype, mask)


@DTYPES
@PAIRS
@pytest.mark.parametrize("mask", [0, 1])
@pytest.mark.parametrize("D", [64, 90])
def test_rotation_alone(D, mask, pairs, dtype):
    case(50, 4, 2, D, D - 10, pairs, dtype, mask, norm=False)


@DTYPES
@PAIRS
def test_far_positions(pairs, dtype):
    """Angles of 10^9, whose 32-bit form would be off by whole turns."""
    case(60, 2, 1, 64, 64, pairs, dtype, far=2 ** 31 - 1, seed=3)


def test_without_scales():
    x, gq, gk, gy, pos = inputs(20, 5, 64, "f32")
    freq = ms.rotary_frequencies(64, device="cuda")
    for a, b, mask in ((None, gk, 5), (gq, None, 3), (None, None, 1)):
        refs, bars = reference(x, a, b, gy, pos, freq, 3, True, False, "f32")
        compare(run(ms.HeadNormRotary(pos, freq, 3), x, a, b, gy, mask), refs, bars, mask)


def test_no_rows():
    x, gq, gk, gy, pos = inputs(0, 5, 64, "bf16")
    y, dx, a, b = run(ms.HeadNormRotary(pos, ms.rotary_frequencies(64, device="cuda"), 3), x, gq, gk, gy, 7)
    assert y.shape == dx.shape == x.shape and not a.any() and not b.any()


def test_keeps_what_the_mask_needs():
    x, gq, gk, gy, pos = inputs(20, 5, 64, "bf16")
    freq = ms.rotary_frequencies(64, device="cuda")
    n = x.numel() * 2
    for mask in range(1, 8):
        live = ms.ledger_read()[0]
        _, rec = ms.layer_forward(ms.HeadNormRotary(pos, freq, 3), x, gq, gk, mask)
        assert rec.account()["saved_activation_bytes"] == ms.ledger_read()[0] - live == n + 80
        assert rec.account()["referenced_param_bytes"] == 128 + (256 if mask & 1 else 0)
        assert set(rec.saved) == {"x", "positions", "inv_freq"} | ({"W", "b"} if mask & 1 else set())
        ms.layer_backward(rec, gy)
        assert ms.ledger_read()[0] == live
    _, rec = ms.layer_forward(ms.HeadNormRotary(pos, freq, 3, norm=False), x, mask=1)
    assert set(rec.saved) == {"positions", "inv_freq"} and rec.account()["saved_activation_bytes"] == 80
    rec.free()


@DTYPES
@PAIRS
@pytest.mark.parametrize("D", [64, 90])
def test_strides(D, pairs, dtype):
    """Views of a projection, heads before rows, elements apart, odd places; results inside larger tensors."""
    T = 33
    _, gq, gk, _, pos = inputs(T, 5, D, dtype)
    p, gy = draw((T, 8, D), dtype, 5), draw((1, 5, D), dtype, 6).expand(T, 5, D)
    x = p[:, 1:6]
    freq = ms.rotary_frequencies(D - 2, device="cuda")
    refs, bars = reference(x, gq, gk, gy, pos, freq, 3, True, pairs, dtype)
    spec = ms.HeadNormRotary(pos, freq, 3, eps=EPS, interleaved=pairs)
    heads = x.transpose(0, 1).contiguous().transpose(0, 1)
    apart = torch.empty(T, 5, 2 * D, dtype=x.dtype, device="cuda")[:, :, ::2].copy_(x)
    odd = torch.empty(T, 5 * D + 3, dtype=x.dtype, device="cuda")[:, 1:1 + 5 * D].unflatten(1, (5, D)).copy_(x)
    for a in (x, heads, apart, odd):
        big, wide = torch.zeros(T, 7, D, dtype=x.dtype, device="cuda"), torch.zeros(T, 5, 2 * D, dtype=x.dtype, device="cuda")
        y, rec = ms.layer_forward(spec, a, gq, gk, 7, y=big[:, 1:6])
        out = ms.layer_backward(rec, gy, wide[:, :, 1::2])
        compare([y] + list(out), refs, bars)
        assert not big[:, 0].any() and not big[:, 6].any() and not wide[:, :, ::2].any()


@DTYPES
@PAIRS
@pytest.mark.parametrize("D,R", [(64, 64), (90, 36), (33, 30)])
def test_in_place(D, R, pairs, dtype):
    x, gq, gk, _, pos = inputs(40, 6, D, dtype)
    spec = ms.HeadNormRotary(pos, ms.rotary_frequencies(R, device="cuda"), 4, interleaved=pairs)
    want = ms.layer_forward(spec, x, gq, gk)[0]
    p = torch.cat([x, x[:, :2]], 1)
    y, _ = ms.layer_forward(spec, p[:, :6], gq, gk, y=p[:, :6])
    assert torch.equal(p[:, :6], want) and torch.equal(p[:, 6:], x[:, :2])
    with pytest.raises(ms.MemsaveError, match="must not be x"):
        ms.layer_forward(spec, x, gq, gk, 1, y=x)
    turn = ms.HeadNormRotary(pos, spec.inv_freq, 4, norm=False, interleaved=pairs)
    want, rec = ms.layer_forward(turn, x, mask=1)
    y, rec2 = ms.layer_forward(turn, x, mask=1, y=x)
    assert torch.equal(x, want) and torch.equal(ms.layer_backward(rec, want)[0], ms.layer_backward(rec2, want)[0])


@DTYPES
@pytest.mark.parametrize("D,R", [(64, 64), (100, 100), (33, 30)])
def test_results_stay_in_their_rows(D, R, dtype):
    x, gq, gk, gy, pos = inputs(21, 5, D, dtype)
    bufs = [guarded_empty((21 * 5, D), dtype) for _ in range(2)]
    _, rec = ms.layer_forward(ms.HeadNormRotary(pos, ms.rotary_frequencies(R, device="cuda"), 3), x, gq, gk, 7, y=bufs[0][0].view(21, 5, D))
    ms.layer_backward(rec, gy, bufs[1][0].view(21, 5, D))
    for view, buf, guard in bufs:
        assert guards_intact(buf, guard) and torch.isfinite(view).all()


@PAIRS
def test_what_does_not_turn_stays(pairs):
    """An infinity beside the turned elements leaves its neighbours alone."""
    x, _, _, _, pos = inputs(9, 2, 64, "f32")
    x[:, :, 33] = math.inf
    y = ms.layer_forward(ms.HeadNormRotary(pos, ms.rotary_frequencies(32, device="cuda"), 1, norm=False, interleaved=pairs), x)[0]
    assert torch.equal(y[:, :, 32:], x[:, :, 32:]) and torch.isfinite(y[:, :, :32]).all()


@DTYPES
def test_same_bits_again_and_in_a_graph(dtype):
    x, gq, gk, gy, pos = inputs(700, 10, 128, dtype)
    spec = ms.HeadNormRotary(pos, ms.rotary_frequencies(128, device="cuda"), 8)
    first = run(spec, x, gq, gk, gy, 7)
    assert all(torch.equal(a, b) for a, b in zip(run(spec, x, gq, gk, gy, 7), first))
    for mask in range(1, 8):
        for a, b in zip(run(spec, x, gq, gk, gy, mask), first):
            assert a is None or torch.equal(a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(spec, x, gq, gk, gy, 7)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(spec, x, gq, gk, gy, 7)
    torch.cuda.synchronize()
    for i in range(3):
        for j, t in enumerate((x, gq, gk, gy)):
            t.copy_(draw(t.shape, dtype, 20 + 10 * i + j))
        pos.add_(17)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, run(spec, x, gq, gk, gy, 7)))


@pytest.mark.parametrize("trains", range(8))
def test_module(trains):
    x, gq, gk, gy, pos = inputs(30, 6, 64, "f32")
    freq = ms.rotary_frequencies(64, device="cuda")
    refs, bars = reference(x, gq, gk, gy, pos, freq, 4, True, False, "f32")
    m = msa.MSHeadNormRotary(gq, gk, 4, freq)
    leaves = [x, m.weight_q, m.weight_k]
    for i, t in enumerate(leaves):
        t.requires_grad_(bool(trains >> i & 1))
    y = m(x, pos)
    if trains:
        y.backward(gy)
    compare([y.detach()] + [t.grad for t in leaves], refs, bars, trains)
    assert not [k for k in m.state_dict() if "freq" in k]


def test_gradients_against_differences():
    """(h = 2^-5 on a unit direction: h^2 / 6 of the third derivative and 2^-24 / h of the
    function are both below 1e-3 of the gradient.)"""
    x, gq, gk, gy, pos = inputs(12, 3, 32, "f32", seed=4)
    spec = ms.HeadNormRotary(pos, ms.rotary_frequencies(32, device="cuda"), 2)
    grads = run(spec, x, gq, gk, gy, 7)[1:]
    f = lambda: (ms.layer_forward(spec, x, gq, gk)[0].double() * gy.double()).sum().item()  # noqa: E731
    gen = torch.Generator().manual_seed(7)
    for t, d in zip((x, gq, gk), grads):
        way = torch.randn(t.shape, generator=gen).cuda()
        way /= way.norm()
        old = t.clone()
        t.copy_(old + 2.0 ** -5 * way)
        up = f()
        t.copy_(old - 2.0 ** -5 * way)
        down = f()
        t.copy_(old)
        assert abs((up - down) * 16 - (d.double() * way.double()).sum().item()) <= 2e-3 * d.norm().item()
