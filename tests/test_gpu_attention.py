"""Attention over whole prompts, forward and backward, against the formulas in 64 bits.

Bars are elementwise and follow the roundings.  With u half a step of the type (2^-8 in
bf16, 2^-24 in fp32) and sums of n terms in fp32 off by at most n 2^-24 of the sum of
their absolute values:
  scores      e = scale (D + 4) 2^-24 sum |q||k| + 2^-21 (the exponential), so P is off by 2 e + n 2^-24 of itself
  o           u |o| + w sum P |v|,  w = u (P as an operand; 0 in fp32) + 2 e + n 2^-24
  dv          u |dv| + w sum P |g|
  delta       sum |g| (error of o) + D 2^-24 sum |g||o|
  dP          D 2^-24 sum |g||v|
  dS          w (|P| (|dP| + |delta|)) + P (errors of dP and delta)
  dq, dk      u |dq| + scale sum (error of dS + (n + 1) 2^-24 |dS|) |k|
All terms below the first order are covered by a factor of 1.05.
"""
import math

import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from _gpu import MARGINS, TORCH_DT, guarded_empty, guards_intact

pytestmark = pytest.mark.gpu
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def draw(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TORCH_DT[dtype]).cuda()


def spans(q_lens, k_lens):
    a = b = 0
    for m, n in zip(q_lens, k_lens):
        yield a, m, b, n
        a, b = a + m, b + n


def starts(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def sequence(q, k, v, g, causal, scale, u):
    """One head of one sequence in 64 bits: results and what each may be off by."""
    m, n, D = q.shape[0], k.shape[0], q.shape[1]
    t = 2.0 ** -24
    if n == 0 or m == 0:
        z = [torch.zeros_like(x) for x in (q, q, k, v)]
        return z, z
    s = scale * (q @ k.t())
    see = torch.ones(m, n, dtype=torch.bool, device=q.device)
    if causal:
        see = see.tril(n - m)
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(1, keepdim=True)
    p = torch.where(see, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
    some = see.any(1, keepdim=True)
    p = torch.where(some, p / torch.where(some, p.sum(1, keepdim=True), 1.0), 0.0)
    e = scale * (D + 4) * t * (q.abs() @ k.abs().t()).max() + 2.0 ** -21
    w = (u if u > 2.0 ** -20 else 0.0) + 2 * e + n * t
    o = p @ v
    bo = u * o.abs() + w * (p @ v.abs())
    dv = p.t() @ g
    bv = u * dv.abs() + (w + m * t) * (p.t() @ g.abs())
    dp = g @ v.t()
    delta = (g * o).sum(1, keepdim=True)
    ds = p * (dp - delta)
    b_delta = (g.abs() * bo).sum(1, keepdim=True) + D * t * (g.abs() * o.abs()).sum(1, keepdim=True)
    bs = p * (w * (dp - delta).abs() + b_delta + D * t * (g.abs() @ v.abs().t()) + 4 * t * (dp.abs() + delta.abs()))
    bs = bs + u * ds.abs() if u > 2.0 ** -20 else bs
    dq, dk = scale * (ds @ k), scale * (ds.t() @ q)
    bq = u * dq.abs() + scale * ((bs + (n + 1) * t * ds.abs()) @ k.abs())
    bk = u * dk.abs() + scale * ((bs + (m + 1) * t * ds.abs()).t() @ q.abs())
    return [o, dq, dk, dv], [bo, bq, bk, bv]


def reference(q, k, v, g, q_lens, k_lens, causal, scale, dtype):
    Hq, Hk = q.shape[1], k.shape[1]
    q, k, v, g = (x.double() for x in (q, k, v, g))
    outs = [torch.zeros_like(x) for x in (q, q, k, v)]
    bars = [torch.zeros_like(x) for x in outs]
    for a, m, b, n in spans(q_lens, k_lens):
        for h in range(Hq):
            c = h * Hk // Hq
            r, e = sequence(q[a:a + m, h], k[b:b + n, c], v[b:b + n, c], g[a:a + m, h], causal, scale, U[dtype])
            for i, (x, y) in enumerate(zip(r, e)):
                rows, head = (slice(a, a + m), h) if i < 2 else (slice(b, b + n), c)
                outs[i][rows, head] += x
                bars[i][rows, head] += y
    return outs, bars


def close(name, got, ref, bar, room=1.05):
    if ref.numel() == 0:
        assert got.shape == ref.shape
        return
    err = (got.double() - ref).abs()
    assert torch.isfinite(err).all(), name
    share = (err / (bar * room + 1e-30)).max().item()
    import os
    MARGINS.append((os.environ.get("PYTEST_CURRENT_TEST", "?").split(" ")[0], name, share, 1.0))
    assert share <= 1.0, f"{name}: {share:.3f} of the bar, error {err.max().item():.3e}"


def run(q, k, v, g, mask, spec, o=None):
    y, rec = ms.layer_forward(spec, q, k, v, mask, y=o)
    return [y] + list(ms.layer_backward(rec, g) if mask else (None,) * 3)


def compare(outs, refs, bars, mask=7):
    for i, name in enumerate(("o", "dq", "dk", "dv")):
        if i and not mask >> (i - 1) & 1:
            assert outs[i] is None
            continue
        close(name, outs[i], refs[i], bars[i])


def case(q_lens, k_lens, Hq, Hk, D, dtype, causal, mask=7, seed=0, std=1.0, packed=True):
    Tq, Tk = sum(q_lens), sum(k_lens)
    q, k, v, g = draw((Tq, Hq, D), dtype, seed, std), draw((Tk, Hk, D), dtype, seed + 1, std), draw((Tk, Hk, D), dtype, seed + 2), draw(
        (Tq, Hq, D), dtype, seed + 3)
    spec = ms.Attention(starts(q_lens) if packed else None, starts(k_lens) if packed and k_lens != q_lens else None, causal=causal)
    refs, bars = reference(q, k, v, g, q_lens, k_lens, causal, D ** -0.5, dtype)
    compare(run(q, k, v, g, mask, spec), refs, bars, mask)


DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])
CAUSAL = pytest.mark.parametrize("causal", [True, False])


@DTYPES
@CAUSAL
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 300])
def test_lengths(n, causal, dtype):
    case([n], [n], 2, 1, 64, dtype, causal, packed=False)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [1, 3, 8, 16, 20, 36, 40, 63, 64, 65, 72, 80, 96, 100, 127, 128, 129, 160, 192, 200, 255, 256])
def test_head_sizes(D, causal, dtype):
    case([70, 5, 131], [70, 5, 131], 2, 1, D, dtype, causal, seed=D)


@DTYPES
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (5, 5), (8, 2), (6, 2), (7, 1), (33, 1), (40, 8)])
def test_grouped_heads(Hq, Hk, dtype):
    case([45, 90], [45, 90], Hq, Hk, 48, dtype, True, seed=Hq)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens", [([1], [1000]), ([130], [131]), ([130], [700]), ([3, 0, 200, 1], [10, 7, 200, 0]),
                                           ([200, 40], [30, 300]), ([0], [50]), ([64, 64], [64, 64])])
def test_keys_of_other_lengths(q_lens, k_lens, D, causal, dtype):
    """Keys before the first query; fewer keys than queries, whose first rows then see none; no
    queries, no keys."""
    case(q_lens, k_lens, 4, 2, D, dtype, causal, seed=11)


@pytest.mark.parametrize("mask", range(8))
@DTYPES
@pytest.mark.parametrize("D", [64, 128, 256])
def test_masks(D, mask, dtype):
    case([100, 37], [100, 37], 4, 2, D, dtype, True, mask, seed=5)


@DTYPES
def test_many_sequences(dtype):
    """More than one wave looks at once; slots that no tile fills."""
    lens = [(7 * i) % 23 for i in range(150)] + [140]
    case(lens, lens, 2, 2, 32, dtype, True, seed=8)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [64, 128])
def test_long(D, causal, dtype):
    case([2500, 1100], [2500, 1100], 2, 1, D, dtype, causal, seed=3)


@CAUSAL
@pytest.mark.parametrize("D", [40, 64, 96, 120, 128])
@pytest.mark.parametrize("q_lens,k_lens", [([2903], [2903]), ([1601], [3333]), ([2903, 1, 0, 1700], [2903, 70, 33, 1600])])
def test_long_walks_of_few_blocks(q_lens, k_lens, D, causal):
    """Blocks whose waves take every other step of the other side."""
    case(q_lens, k_lens, 16, 8, D, "bf16", causal, seed=5)


@CAUSAL
@pytest.mark.parametrize("q_lens,k_lens", [([3500], [3500]), ([1800], [5000])])
def test_long_walks_divided(q_lens, k_lens, causal):
    """The same where the keys are divided over blocks as well."""
    case(q_lens, k_lens, 8, 4, 64, "bf16", causal, seed=6)


@pytest.mark.parametrize("D", [64, 128])
def test_long_walks_by_mask(D):
    q, k, v, g = (draw((2903, h, D), "bf16", i) for i, h in enumerate((16, 8, 8, 16)))
    first = run(q, k, v, g, 7, ms.Attention())
    for mask in range(1, 8):
        for a, b in zip(run(q, k, v, g, mask, ms.Attention()), first):
            assert a is None or torch.equal(a, b)
    # keys that are not finite: the rows before them are as without, but for the order of sums in
    # tiles that hold some (a row of the tile after the other), so as near to the reference
    at = 1500
    refs, bars = reference(q, k, v, g, [2903], [2903], True, D ** -0.5, "bf16")
    for which in range(2):
        k2, v2 = k.clone(), v.clone()
        (k2, v2)[which][at:] = math.nan
        outs = run(q, k2, v2, g, 7, ms.Attention())
        for i in (0, 1):
            close("od"[i], outs[i][:at], refs[i][:at], bars[i][:at])
        assert torch.isnan(outs[0][at:].float()).all()


@DTYPES
def test_large_scores(dtype):
    """Rows near one-hot: the running maximum moves, probabilities underflow."""
    case([300], [300], 2, 1, 64, dtype, True, std=6.0, seed=4)


@DTYPES
def test_growing_scores(dtype):
    """Each key's score above the one before it: the reference moves at every step."""
    n, D = 400, 64
    q = torch.ones(n, 1, D, dtype=TORCH_DT[dtype], device="cuda")
    k = (torch.arange(n, device="cuda") / 8.0).to(TORCH_DT[dtype])[:, None, None].expand(n, 1, D).contiguous()
    v, g = draw((n, 1, D), dtype, 1), draw((n, 1, D), dtype, 2)
    refs, bars = reference(q, k, v, g, [n], [n], True, D ** -0.5, dtype)
    compare(run(q, k, v, g, 7, ms.Attention()), refs, bars)


@DTYPES
def test_keeps_what_the_mask_needs(dtype):
    q, k, v, g = draw((70, 4, 64), dtype, 1), draw((70, 2, 64), dtype, 2), draw((70, 2, 64), dtype, 3), draw((70, 4, 64), dtype, 4)
    off = starts([30, 40])
    nq, nk = q.numel() * q.element_size(), k.numel() * k.element_size()
    for mask in range(1, 8):
        live = ms.ledger_read()[0]
        y, rec = ms.layer_forward(ms.Attention(off), q, k, v, mask)
        both = bool(mask & 3)
        assert rec.account()["saved_activation_bytes"] == ms.ledger_read()[0] - live == nq + nk + 70 * 4 * 4 + 3 * 4 + both * (nk + nq)
        assert set(rec.saved) == {"x", "W", "lse", "offsets"} | ({"v", "o"} if both else set())
        ms.layer_backward(rec, g)
        assert ms.ledger_read()[0] == live
    assert ms.layer_forward(ms.Attention(off), q, k, v, 0)[1] is None


@DTYPES
@pytest.mark.parametrize("D", [64, 128, 200])
def test_rows_of_no_sequence(D, dtype):
    """Before the first and past the last: zeros, whatever they hold and whatever was there."""
    q, k, v, g = (draw((200, h, D), dtype, i) for i, h in enumerate((4, 2, 2, 4)))
    lens = [50, 60]
    off = starts(lens) + 20
    refs, bars = reference(q[20:130], k[20:130], v[20:130], g[20:130], lens, lens, True, D ** -0.5, dtype)
    for t in (q, k, v, g):
        t[:20], t[130:] = math.nan, math.inf
    o = torch.full_like(q, math.nan)
    outs = run(q, k, v, g, 7, ms.Attention(off), o)
    for t in outs:
        assert not t[:20].any() and not t[130:].any()
    compare([t[20:130] for t in outs], refs, bars)


@DTYPES
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_places_hold_anything(bad, D, dtype):
    """A key, a value or a query that is not finite: rows that do not see it are as without it."""
    n, at = 150, 77
    q, k, v, g = (draw((n, 2, D), dtype, i) for i in range(4))
    refs, bars = reference(q, k, v, g, [n], [n], True, D ** -0.5, dtype)
    spec = ms.Attention()
    for which in range(2):   # a key and its value: later rows see them
        k2, v2 = k.clone(), v.clone()
        (k2, v2)[which][at] = bad
        outs = run(q, k2, v2, g, 7, spec)
        for i in (0, 1):
            close("od"[i], outs[i][:at], refs[i][:at], bars[i][:at])
        assert not torch.isfinite(outs[0][at:].float()).all()
    # a query's row and its gradient's: keys past it do not enter into them
    for which in range(2):
        q2, g2 = q.clone(), g.clone()
        (q2, g2)[which][at] = bad
        outs = run(q2, k, v, g2, 7, spec)
        for i in (0, 1):
            keep = torch.arange(n, device="cuda") != at
            close("od"[i], outs[i][keep], refs[i][keep], bars[i][keep])
        for i in (2, 3):
            close("kv"[i - 2], outs[i][at + 1:], refs[i][at + 1:], bars[i][at + 1:])


@DTYPES
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 40, 64, 150])
def test_a_key_that_no_query_weighs(n, D, dtype):
    """Scores of minus infinity with one key, from every query: its gradients are 0, all
    others as without it (rows past the last query add nothing to it)."""
    keys, at = 90, 41
    q, k, v, g = draw((n, 2, D), dtype, 0), draw((keys, 2, D), dtype, 1), draw((keys, 2, D), dtype, 2), draw((n, 2, D), dtype, 3)
    q[:, :, 0] = 1.0
    k[:, :, 0] = 0.0
    rest = torch.arange(keys, device="cuda") != at
    refs, bars = reference(q, k[rest], v[rest], g, [n], [keys - 1], False, D ** -0.5, dtype)
    k[at, :, 0] = -math.inf
    o, _, dk, dv = run(q, k, v, g, 6, ms.Attention(causal=False))
    assert (dk[at] == 0).all() and (dv[at] == 0).all()
    for name, got, i in (("o", o, 0), ("k", dk[rest], 2), ("v", dv[rest], 3)):
        close(name, got, refs[i], bars[i])


def test_scores_without_a_distribution():
    """All visible scores minus infinity, or one plus infinity: NaN; a single minus infinity: left out."""
    D = 64
    q = torch.zeros(3, 1, D, device="cuda")
    q[:, :, 0] = 1.0
    k, v = torch.zeros(3, 1, D, device="cuda"), draw((3, 1, D), "f32", 1)
    k[0, 0, 0] = -math.inf
    o = ms.layer_forward(ms.Attention(), q, k, v)[0]
    assert torch.isnan(o[0]).all() and torch.allclose(o[1], v[1]) and torch.isfinite(o[2]).all()
    k[0, 0, 0] = math.inf
    assert torch.isnan(ms.layer_forward(ms.Attention(), q, k, v)[0]).all()


@DTYPES
@pytest.mark.parametrize("D", [64, 100, 128])
def test_strides(D, dtype):
    """Views of one projection (in place), heads before rows, elements apart, expanded gradients; results inside
    larger tensors."""
    n, lens = 150, [60, 90]
    p = draw((n, 8, D), dtype, 1)
    q, k, v = p[:, :4], p[:, 4:6], p[:, 6:]
    g = draw((1, 1, D), dtype, 2).expand(n, 4, D)
    refs, bars = reference(q, k, v, g, lens, lens, True, D ** -0.5, dtype)
    spec = ms.Attention(starts(lens))
    y, rec = ms.layer_forward(spec, q, k, v, 7)
    assert rec.saved["x"] is q
    compare([y] + list(ms.layer_backward(rec, g)), refs, bars)
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    apart = [torch.empty(n, x.shape[1], 2 * D, dtype=x.dtype, device="cuda")[:, :, ::2].copy_(x) for x in (q, k, v)]
    odd = [torch.empty(n, x.shape[1] * D + 3, dtype=x.dtype, device="cuda")[:, 1:1 + x.shape[1] * D].unflatten(1, (x.shape[1], D)).copy_(x) for x in (q, k, v)]
    for a, b, c in (turned, apart, odd):
        big = torch.zeros(n, 10, D, dtype=p.dtype, device="cuda")
        y, rec = ms.layer_forward(spec, a, b, c, 7, y=big[:, 3:7])
        grads = torch.zeros(n, 9, D, dtype=p.dtype, device="cuda")
        out = ms.layer_backward(rec, g, grads[:, :4], grads[:, 4:6], grads[:, 7:])
        compare([y] + list(out), refs, bars)
        assert not big[:, :3].any() and not big[:, 7:].any() and not grads[:, 6].any()


@DTYPES
@pytest.mark.parametrize("D", [64, 72, 128, 256])
def test_results_stay_in_their_rows(D, dtype):
    n = 77
    q, k, v, g = (draw((n, 2, D), dtype, i) for i in range(4))
    bufs = [guarded_empty((n * 2, D), dtype) for _ in range(4)]
    views = [b[0].view(n, 2, D) for b in bufs]
    y, rec = ms.layer_forward(ms.Attention(), q, k, v, 7, y=views[0])
    ms.layer_backward(rec, g, *views[1:])
    for view, buf, guard in bufs:
        assert guards_intact(buf, guard) and torch.isfinite(view).all()


def test_one_row_of_any_stride():
    """A tensor of one row may state any stride for it."""
    q, k, v = (draw((1, 2, 64), "bf16", i) for i in range(3))
    ref = ms.layer_forward(ms.Attention(), q, k, v)[0]
    q, k, v = (x.as_strided((1, 2, 64), (3, 64, 1)) for x in (q, k, v))
    assert torch.equal(ms.layer_forward(ms.Attention(), q, k, v)[0], ref) and torch.equal(ref, v)


@DTYPES
def test_same_bits_again(dtype):
    q, k, v, g = (draw((700, h, 128), dtype, i) for i, h in enumerate((8, 2, 2, 8)))
    spec = ms.Attention(starts([300, 400]))
    first = run(q, k, v, g, 7, spec)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(q, k, v, g, 7, spec), first))
    # what the mask leaves out changes nothing of the rest
    for mask in range(1, 8):
        for a, b in zip(run(q, k, v, g, mask, spec), first):
            assert a is None or torch.equal(a, b)


@DTYPES
def test_graph_replays(dtype):
    """Forward and backward in a graph, replayed on other inputs, with eager calls between."""
    q, k, v, g = (draw((260, h, 96), dtype, i) for i, h in enumerate((4, 2, 2, 4)))
    spec = ms.Attention(starts([60, 200]))
    run(q, k, v, g, 7, spec)   # (the workspace)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(q, k, v, g, 7, spec)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(q, k, v, g, 7, spec)
    torch.cuda.synchronize()
    for i in range(4):
        for j, t in enumerate((q, k, v, g)):
            t.copy_(draw(t.shape, dtype, 10 * i + j + 50))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, run(q, k, v, g, 7, spec)))


@DTYPES
def test_graph_replays_of_other_sequences(dtype):
    """The offsets are read by the kernels: a replay has the sequences that they then name."""
    T, D = 700, 64
    q, k, v, g = (draw((T, h, D), dtype, i) for i, h in enumerate((4, 2, 2, 4)))
    off = starts([100, 300, 300])
    spec = ms.Attention(off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(q, k, v, g, 7, spec)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(q, k, v, g, 7, spec)
    torch.cuda.synchronize()
    for lens in ([700, 0, 0], [1, 698, 1], [200, 33, 7], [0, 0, 0], [100, 300, 300]):
        off.copy_(starts(lens))
        for t in outs:
            t.fill_(7.0)   # (all rows are written, also those of no sequence)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, run(q, k, v, g, 7, spec)))
        assert (outs[0][sum(lens):] == 0).all() and all(torch.isfinite(t.float()).all() for t in outs)


def test_threads():
    """Calls of several threads, on one stream and on streams of their own."""
    import threading
    shapes = [(700, 4, 2, 64), (2903, 16, 8, 128), (90, 2, 1, 100), (1300, 6, 2, 72)]
    data = [[draw((T, h, D), "bf16" if i % 2 else "f32", 10 * i + j) for j, h in enumerate((Hq, Hk, Hk, Hq))]
            for i, (T, Hq, Hk, D) in enumerate(shapes)]
    want = [run(*t, 7, ms.Attention()) for t in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.current_stream()] * 2 + [torch.cuda.Stream() for _ in range(2)]
    bad = []

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(5):
                got = run(*data[i], 7, ms.Attention())
                streams[i].synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@DTYPES
def test_broadcast_inputs(dtype):
    """A head of keys and values that all heads share by a stride of 0: its gradient is the sum over them."""
    T, D = 200, 64
    q, g = draw((T, 4, D), dtype, 0), draw((T, 4, D), dtype, 3)
    k1, v1 = draw((T, 1, D), dtype, 1).requires_grad_(), draw((T, 1, D), dtype, 2).requires_grad_()
    msa.MSAttention()(q, k1.expand(T, 4, D), v1.expand(T, 4, D)).backward(g)
    refs, bars = reference(q, k1.detach(), v1.detach(), g, [T], [T], True, D ** -0.5, dtype)
    for name, got, i in (("k", k1.grad, 2), ("v", v1.grad, 3)):
        # four gradients, each rounded once, and the roundings of their sum
        close(name, got, refs[i], 4 * bars[i])


def test_on_another_stream():
    q, k, v, g = (draw((300, 2, 80), "bf16", i) for i in range(4))
    first = run(q, k, v, g, 7, ms.Attention())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y, rec = ms.layer_forward(ms.Attention(), q, k, v, 7)
    torch.cuda.current_stream().wait_stream(s)
    grads = ms.layer_backward(rec, g)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip([y] + list(grads), first))


def test_without_allocation():
    """ms_layer_backward_noalloc: the same bits."""
    import ctypes
    from paper_2404_12406_amd import _lib, api
    q, k, v, g = (draw((200, 2, 72), "bf16", i) for i in range(4))
    first = run(q, k, v, g, 7, ms.Attention())
    _, rec = ms.layer_forward(ms.Attention(), q, k, v, 7)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    st = _lib.load().ms_layer_backward_noalloc(rec._h, *(ctypes.byref(api.tensor_desc(t)) for t in [g] + grads), api._stream(q.device))
    assert st == 0
    assert all(torch.equal(a, b) for a, b in zip(grads, first[1:]))


@pytest.mark.parametrize("trains", range(1, 8))
def test_module(trains):
    q, k, v, g = (draw((120, h, 64), "f32", i) for i, h in enumerate((4, 2, 2, 4)))
    for i, t in enumerate((q, k, v)):
        t.requires_grad_(bool(trains >> i & 1))
    lens = [50, 70]
    m = msa.MSAttention()
    y = m(q, k, v, starts(lens))
    y.backward(g)
    refs, bars = reference(q.detach(), k.detach(), v.detach(), g, lens, lens, True, 0.125, "f32")
    compare([y, q.grad, k.grad, v.grad], refs, bars, trains)
    with torch.no_grad():
        assert torch.equal(m(q, k, v, starts(lens)), y)


def test_gradients_against_differences():
    """Of a sum of o's elements by weights, in fp32 (128 bits of headroom: h = 2^-5, the third
    derivative's part h^2 / 6 and rounding 2^-24 / h are both below 1e-3 of the largest gradient)."""
    q, k, v, g = (draw((40, h, 32), "f32", i, 0.5) for i, h in enumerate((4, 2, 2, 4)))
    grads = run(q, k, v, g, 7, ms.Attention())[1:]
    h = 2.0 ** -5
    f = lambda: (ms.layer_forward(ms.Attention(), q, k, v)[0].double() * g.double()).sum().item()  # noqa: E731
    gen = torch.Generator().manual_seed(7)
    for t, d in zip((q, k, v), grads):
        way = torch.randn(t.shape, generator=gen).cuda()
        way /= way.norm()
        old = t.clone()
        t.copy_(old + h * way)
        up = f()
        t.copy_(old - h * way)
        down = f()
        t.copy_(old)
        want = (d.double() * way.double()).sum().item()
        assert abs((up - down) / (2 * h) - want) <= 2e-3 * d.norm().item()


def test_modified_in_place_and_twice():
    q, k, v = (draw((40, 2, 64), "f32", i).requires_grad_() for i in range(3))
    y = msa.MSAttention()(q, k, v)
    with torch.no_grad():
        v.add_(1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()
    y = msa.MSAttention()(q, k, v)
    y.sum().backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="second time"):
        y.sum().backward()


def test_an_unused_output_is_released():
    """A record holds its own output, but no cycle through it."""
    import gc
    q, k, v = (draw((64, 2, 64), "f32", i).requires_grad_() for i in range(3))
    live = ms.ledger_read()[0]
    gc.disable()
    try:
        y = msa.MSAttention()(q, k, v)
        assert ms.ledger_read()[0] > live
        del y
        assert ms.ledger_read()[0] == live
    finally:
        gc.enable()
