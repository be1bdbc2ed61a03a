"""The paged cache and the attention of single tokens over it, against the formulas in 64
bits (bars as in test_gpu_attention.py), and a run of the attention's operators together."""
import math

import pytest
import torch

import paper_2404_12406_amd as ms
from _gpu import TORCH_DT
from test_gpu_attention import close, draw, reference, starts
from test_gpu_head_norm_rotary import inputs

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Cache:
    """Pages in no order; what no sequence uses holds NaN."""

    def __init__(self, lengths, Hk, D, page, dtype, seed=0, spare=2, width=None):
        gen = torch.Generator().manual_seed(seed)
        need = [-(-max(n, 0) // page) for n in lengths]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=gen).tolist()
        width = max(need + [1]) if width is None else width
        # (past what a sequence needs: pages that do not exist)
        self.tables = ints([[order.pop() if i < m else (-1, pages, 2 ** 31 - 1)[i % 3] for i in range(width)] for m in need])
        self.k = torch.full((pages, Hk, page, D), math.nan, dtype=TORCH_DT[dtype], device="cuda")
        self.v = self.k.clone()
        self.lengths, self.page = ints(lengths), page
        self.keys, self.values = [], []
        for b, n in enumerate(lengths):
            k, v = draw((max(n, 0), Hk, D), dtype, seed + 2 * b + 1), draw((max(n, 0), Hk, D), dtype, seed + 2 * b + 2)
            self.keys.append(k)
            self.values.append(v)
            at = torch.arange(max(n, 0), device="cuda")
            if n > 0:
                pg = self.tables[b].long()[at // page]
                self.k[pg, :, at % page] = k
                self.v[pg, :, at % page] = v

    def attend(self, q, **kw):
        return ms.layer_forward(ms.PagedAttention(self.k, self.v, self.tables, self.lengths, **kw), q)[0]


def check(c, q, o, dtype, scale=None):
    lens = [max(n, 0) for n in c.lengths.tolist()]
    refs, bars = reference(q, torch.cat(c.keys), torch.cat(c.values), torch.zeros_like(q), [1] * len(lens), lens, False,
                           q.shape[2] ** -0.5 if scale is None else scale, dtype)
    close("o", o, refs[0], bars[0])


def case(lengths, Hq, Hk, D, page, dtype, seed=0, **kw):
    c = Cache(lengths, Hk, D, page, dtype, seed, **kw)
    q = draw((len(lengths), Hq, D), dtype, seed + 99)
    check(c, q, c.attend(q), dtype)


@DTYPES
@pytest.mark.parametrize("page", [1, 5, 16, 24, 32, 64, 100, 128])
def test_page_sizes(page, dtype):
    case([1, 31, 32, 33, 127, 128, 129, 200, 0, 700], 4, 2, 64, page, dtype, page)


@DTYPES
@pytest.mark.parametrize("D", [1, 3, 8, 16, 36, 63, 64, 72, 80, 100, 127, 128, 129, 145, 200, 255, 256])
def test_head_sizes(D, dtype):
    case([300, 40, 1], 6, 2, D, 16, dtype, D)


@DTYPES
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (8, 8), (15, 3), (32, 1), (33, 1), (80, 2), (40, 8)])
def test_grouped_heads(Hq, Hk, dtype):
    case([150, 290], Hq, Hk, 128, 16, dtype, Hq)


@DTYPES
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long(D, dtype):
    """Several steps of every wave of a block, several blocks a sequence."""
    case([9000, 2, 4097, 640], 4, 1, D, 64, dtype, 1)
    case([6000] * 40, 2, 1, D, 16, dtype, 2)


@DTYPES
def test_a_wide_table(dtype):
    """Room for far more places than are used."""
    case([100, 5000, 1], 4, 2, 64, 16, dtype, 3, width=20000)


@DTYPES
def test_lengths_that_are_none(dtype):
    """Nothing and less: zeros.  More than the table holds, or a page outside the cache: NaN, for that sequence alone."""
    c = Cache([40, 50, 60, 70, 80], 2, 64, 16, dtype)
    q = draw((5, 4, 64), dtype, 7)
    good = c.attend(q)
    c.lengths = ints([0, -5, c.tables.shape[1] * 16 + 1, 70, 80])
    c.tables[4, 2] = c.k.shape[0]
    o = c.attend(q)
    assert not o[:2].any() and torch.isnan(o[2]).all() and torch.equal(o[3], good[3]) and torch.isnan(o[4]).all()
    c.tables[4, 2] = -1
    c.tables[3, 4] = 2 ** 31 - 1   # its last page of 16, of which 6 places are used
    assert torch.isnan(c.attend(q)[3:]).all()


def test_no_sequences_and_no_pages():
    c = Cache([], 2, 64, 16, "bf16")
    tables = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    q = draw((0, 4, 64), "bf16", 1)
    assert ms.layer_forward(ms.PagedAttention(c.k, c.v, tables, c.lengths), q)[0].shape == (0, 4, 64)
    q = draw((2, 4, 64), "bf16", 1)
    empty = c.k[:0]
    for width, lengths, nan in ((0, [0, 0], [False, False]), (2, [0, 1], [False, True])):
        o = ms.layer_forward(ms.PagedAttention(empty, empty, torch.zeros((2, width), dtype=torch.int32, device="cuda"), ints(lengths)), q)[0]
        assert torch.isnan(o).all(-1).all(-1).tolist() == nan and not o[0].any()


@DTYPES
@pytest.mark.parametrize("D", [64, 100])
def test_strides(D, dtype):
    c = Cache([90, 200, 3], 2, D, 16, dtype)
    p = draw((3, 9, D), dtype, 3)
    q = p[:, 2:8]
    want = c.attend(q.contiguous())
    apart = torch.empty(3, 6, 2 * D, dtype=p.dtype, device="cuda")[:, :, ::2].copy_(q)
    heads = q.transpose(0, 1).contiguous().transpose(0, 1)
    for x in (q, apart, heads):
        big = torch.zeros(3, 8, 2 * D, dtype=p.dtype, device="cuda")
        for y in (big[:, 1:7, :D], big[:, 1:7, ::2]):
            big.zero_()
            ms.layer_forward(ms.PagedAttention(c.k, c.v, c.tables, c.lengths), x, y=y)
            assert torch.equal(y, want)
            y.zero_()
            assert not big.any()


@DTYPES
def test_a_cache_past_32_bit_offsets(dtype):
    """Pages past 2^31 elements, 4 GiB and 8 GiB into the cache: written and read."""
    Hk, page, D = 8, 64, 128
    per = Hk * page * D
    pages = 2 ** 31 // per + 2 ** 31 // per + 9
    k, v = (torch.empty((pages, Hk, page, D), dtype=TORCH_DT[dtype], device="cuda") for _ in range(2))
    ids = [3, 2 ** 31 // per - 1, 2 ** 31 // per, 2 ** 31 // per + 5, pages - 1]
    tables = ints([ids[::-1], ids])
    n = 4 * page + 17
    x = draw((n, 3 * Hk, D), dtype, 1)
    # the second sequence, at its last n - 1 places and its first
    pos = ints([0] + list(range(1, n)))
    q, _ = ms.layer_forward(ms.CacheAppend(k, v, tables, pos, ints([1] * n), q_heads=Hk, norm=False), x)
    assert torch.equal(q, x[:, :Hk])
    for i, pg in enumerate(ids):
        part = x[page * i:min(n, page * i + page)]
        assert torch.equal(k[pg, :, :len(part)].transpose(0, 1), part[:, Hk:2 * Hk])
        assert torch.equal(v[pg, :, :len(part)].transpose(0, 1), part[:, 2 * Hk:])
    lengths = ints([0, n])
    o = ms.layer_forward(ms.PagedAttention(k, v, tables, lengths), x[-2:, :Hk])[0]
    refs, bars = reference(x[-1:, :Hk], x[:, Hk:2 * Hk], x[:, 2 * Hk:], x[-1:, :Hk], [1], [n], False, D ** -0.5, dtype)
    close("o", o[1:], refs[0], bars[0])
    assert not o[0].any()


# ------------------------------------------------------------------ appending
@DTYPES
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("D,R,norm", [(64, 64, True), (128, 128, True), (90, 36, True), (145, 144, True), (64, 0, True), (64, 64, False), (100, 0, False)])
def test_append(D, R, norm, pairs, dtype):
    """Queries and keys as HeadNormRotary's, bit for bit, values as they are, nothing else written."""
    Hq, Hk, page, lens = 6, 2, 16, [40, 1, 33, 0, 100]
    T = sum(lens)
    x, gq, gk, _, _ = inputs(T, Hq + 2 * Hk, D, dtype)
    if not norm:
        gq = gk = None
    c = Cache([n + 7 for n in lens], Hk, D, page, dtype)
    was_k, was_v = c.k.clone(), c.v.clone()
    rows = torch.repeat_interleave(torch.arange(5, device="cuda"), torch.tensor(lens, device="cuda"))
    pos = torch.cat([torch.arange(n) + 7 for n in lens]).cuda()
    freq = ms.rotary_frequencies(R, device="cuda") if R else None
    q, rec = ms.layer_forward(ms.CacheAppend(c.k, c.v, c.tables, pos.int(), rows.int(), freq, Hq, norm, interleaved=pairs), x, gq, gk)
    y = ms.layer_forward(ms.HeadNormRotary(pos.int(), freq, Hq, norm, interleaved=pairs), x[:, :Hq + Hk], gq, gk)[0]
    assert rec is None and torch.equal(q, y[:, :Hq])
    pg = c.tables.long()[rows, pos // page]
    was_k[pg, :, pos % page], was_v[pg, :, pos % page] = y[:, Hq:], x[:, Hq + Hk:]
    for got, want in ((c.k, was_k), (c.v, was_v)):
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want)) and torch.equal(torch.isnan(got), torch.isnan(want))


@DTYPES
def test_tokens_without_a_place(dtype):
    """Positions, sequences and pages that are none: the cache stays, the queries are taken."""
    Hq, Hk, D, page = 2, 1, 64, 16
    c = Cache([20, 20], Hk, D, page, dtype, width=2)
    c.tables[1, 1] = c.k.shape[0]
    was = c.k.clone(), c.v.clone()
    x = draw((7, Hq + 2 * Hk, D), dtype, 1)
    pos, rows = ints([-1, 32, 2 ** 31 - 1, -2 ** 31, 17, 0, 0]), ints([0, 0, 0, 0, 1, 2, -1])
    q, _ = ms.layer_forward(ms.CacheAppend(c.k, c.v, c.tables, pos, rows, q_heads=Hq, norm=False), x)
    assert torch.equal(q, x[:, :Hq])
    for got, want in zip((c.k, c.v), was):
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@DTYPES
def test_keys_and_values_alone(dtype):
    """No queries; a view of a larger tensor; a token a sequence; elements apart."""
    Hk, D, page = 2, 64, 16
    c = Cache([5, 30, 17], Hk, D, page, dtype)
    p = draw((3, 6, D), dtype, 1)
    for x in (p[:, 2:], torch.empty(3, 4, 2 * D, dtype=p.dtype, device="cuda")[:, :, ::2].copy_(p[:, 2:])):
        pos = c.lengths - 1
        y, _ = ms.layer_forward(ms.CacheAppend(c.k, c.v, c.tables, pos, norm=False), x)
        assert y.shape == (3, 0, D)
        at = c.tables.long()[torch.arange(3, device="cuda"), pos.long() // page], pos.long() % page
        assert torch.equal(c.k[at[0], :, at[1]], x[:, :2]) and torch.equal(c.v[at[0], :, at[1]], x[:, 2:])
        c.k.fill_(0), c.v.fill_(0)


def test_one_place_twice():
    """Each 16 bytes are one of the two tokens'."""
    x = draw((2, 2, 64), "bf16", 1)
    k, v = torch.zeros(1, 1, 16, 64, dtype=x.dtype, device="cuda"), torch.zeros(1, 1, 16, 64, dtype=x.dtype, device="cuda")
    ms.layer_forward(ms.CacheAppend(k, v, ints([[0]]), ints([3, 3]), ints([0, 0]), norm=False), x)
    for pages, h in ((k, 0), (v, 1)):
        got = pages[0, 0, 3].view(8, 8)
        assert all(torch.equal(got[i], x[0, h].view(8, 8)[i]) or torch.equal(got[i], x[1, h].view(8, 8)[i]) for i in range(8))


# ------------------------------------------------------------------ together
@DTYPES
@pytest.mark.parametrize("Hq,Hk,D", [(8, 2, 64), (4, 4, 128), (3, 1, 90)])
def test_prompt_and_tokens(Hq, Hk, D, dtype):
    """A prompt through HeadNormRotary, Attention and CacheAppend, then token by token through
    CacheAppend and PagedAttention, in a graph: each token's output is that of the whole
    sequence at once (both within their bars)."""
    prompts, more, page = [37, 1, 90], 6, 16
    total = [n + more for n in prompts]
    _, gq, gk, _, _ = inputs(1, 1, D, dtype)
    freq = ms.rotary_frequencies(D - D % 2, device="cuda")
    x = [draw((n, Hq + 2 * Hk, D), dtype, 10 + b) for b, n in enumerate(total)]
    # whole sequences
    whole = torch.cat(x)
    at = torch.cat([torch.arange(n) for n in total]).int().cuda()
    y = ms.layer_forward(ms.HeadNormRotary(at, freq, Hq), whole[:, :Hq + Hk], gq, gk)[0]
    refs, bars = reference(y[:, :Hq], y[:, Hq:], whole[:, Hq + Hk:], y[:, :Hq], total, total, True, D ** -0.5, dtype)
    o = ms.layer_forward(ms.Attention(starts(total)), y[:, :Hq], y[:, Hq:], whole[:, Hq + Hk:])[0]
    close("whole", o, refs[0], bars[0])
    # the prompts, in place, and then into the cache as they are
    c = Cache(total, Hk, D, page, dtype)
    c.k.fill_(math.nan), c.v.fill_(math.nan)
    p = torch.cat([t[:n] for t, n in zip(x, prompts)])
    pos = torch.cat([torch.arange(n) for n in prompts]).int().cuda()
    ms.layer_forward(ms.HeadNormRotary(pos, freq, Hq), p[:, :Hq + Hk], gq, gk, y=p[:, :Hq + Hk])
    o = ms.layer_forward(ms.Attention(starts(prompts)), p[:, :Hq], p[:, Hq:Hq + Hk], p[:, Hq + Hk:])[0]
    first = [0, total[0], total[0] + total[1]]
    keep = torch.cat([torch.arange(f, f + n) for f, n in zip(first, prompts)]).cuda()
    close("prompts", o, refs[0][keep], bars[0][keep])
    rows = torch.repeat_interleave(torch.arange(3), torch.tensor(prompts)).int().cuda()
    ms.layer_forward(ms.CacheAppend(c.k, c.v, c.tables, pos, rows, norm=False), p[:, Hq:])
    # the tokens
    token, where, lengths = torch.empty(3, Hq + 2 * Hk, D, dtype=p.dtype, device="cuda"), ints(prompts), ints(prompts) + 1

    def step():
        q, _ = ms.layer_forward(ms.CacheAppend(c.k, c.v, c.tables, where, None, freq, Hq), token, gq, gk)
        return ms.layer_forward(ms.PagedAttention(c.k, c.v, c.tables, lengths), q)[0]

    token.copy_(torch.stack([t[n] for t, n in zip(x, prompts)]))
    eager = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = step()
    torch.cuda.synchronize()
    for i in range(more):
        token.copy_(torch.stack([t[n + i] for t, n in zip(x, prompts)]))
        where.copy_(ints(prompts) + i)
        lengths.copy_(where + 1)
        graph.replay()
        torch.cuda.synchronize()
        if i == 0:
            assert torch.equal(out, eager)
        keep = ints([f + n + i for f, n in zip(first, prompts)]).long()
        close("token", out, refs[0][keep], bars[0][keep])
        assert torch.equal(out, step())


def test_graphs_and_eager_calls_share_no_results():
    """Two graphs and eager calls of other sizes on one stream, in turn."""
    cs = [Cache([3000, 500], 2, 128, 16, "bf16", 1), Cache([700, 6000, 20], 2, 128, 16, "bf16", 2)]
    qs = [draw((c.lengths.shape[0], 8, 128), "bf16", 5) for c in cs]
    want = [c.attend(q) for c, q in zip(cs, qs)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(s):
        for c, q in zip(cs, qs):
            c.attend(q)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(c.attend(q))
            graphs.append(g)
        big = Cache([20000] * 3, 2, 128, 16, "bf16", 3)
        big.attend(draw((3, 8, 128), "bf16", 6))   # outgrows the workspace that the graphs hold
        for _ in range(3):
            for g, o, w, c, q in zip(graphs, outs, want, cs, qs):
                o.zero_()
                g.replay()
                again = c.attend(q)
                s.synchronize()
                assert torch.equal(o, w) and torch.equal(again, w)


def test_prepared_calls():
    c = Cache([40, 90], 2, 64, 16, "bf16")
    x = draw((2, 8, 64), "bf16", 1)
    a = ms.PreparedLayer(ms.CacheAppend(c.k, c.v, c.tables, c.lengths - 1, q_heads=4, norm=False), x)
    a.forward()
    b = ms.PreparedLayer(ms.PagedAttention(c.k, c.v, c.tables, c.lengths), a.y)
    b.forward()
    assert torch.equal(a.y, x[:, :4]) and torch.equal(b.y, c.attend(x[:, :4]))
