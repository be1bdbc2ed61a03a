"""The attention of a transformer block -- head norms with the position rotation, attention over
whole prompts, a paged cache and the attention of single tokens over it -- as measurable cases.

One pass is one operator as a program calls it: the forward alone where nothing asks for a
gradient (prompts, tokens), else the forward and the backward that writes exactly the gradients
the mask asks for.  The plain form is the same mathematics in elementary torch operations, in 32
bits (angles in 64), rounded once at the end; `exact` is the definition again in 64 bits.

    rotary   z = x / sqrt(mean x^2 + eps) * g over each head of x[T, Hq + Hk, D], g = gq for the first Hq
             heads and gk for the others; the first R of its D elements then turn in pairs, (i, i + R/2) or
             (2 i, 2 i + 1), by the angle position * freq[i]
    attend   o = softmax(scale q k^T) v for each of several packed sequences and each head, Hq / Hk
             query heads to a head of k and v; causal: the last query sees every key, the one before
             it all but one
    append   rotary of the q and k heads of x[T, Hq + Hk + Hk, D]; k and v then go to their places in a
             cache of pages [pages, Hk, page, D] by each token's sequence and position
    paged    o = softmax(scale q k^T) v of one query a sequence over the first length[b] places of its
             pages, which table[b] lists
"""
import math
import random

import torch

own = False   # plain form (False) or the library's kernels (True)

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ELT = {"f32": 4, "bf16": 2}
EPS = 1e-6
THETA = 10000.0


def listed():
    return [
        # Four requests' new tokens through the head norms of a layer: launch latency is all of it.
        dict(name="rotary_token_bf16", op="rotary", dtype="bf16", t=4, hq=32, hk=8, d=128, r=128, pairs=False, far=30000, mask=0),
        # A training batch of 16 x 512 tokens, scales trained.
        dict(name="rotary_train_bf16", op="rotary", dtype="bf16", t=8192, hq=32, hk=8, d=128, r=128, pairs=False, far=512, mask=7),
        # float32, rows that no vector divides, neighbours in pairs, a part of each head turned, positions far out.
        dict(name="rotary_ragged_f32", op="rotary", dtype="f32", t=3001, hq=10, hk=5, d=90, r=36, pairs=True, far=1000000, mask=7),
        # The encoder's attention: 16 x 512 tokens, hidden size 768 in heads of 64, everything trained.
        dict(name="attend_train_bf16", op="attend", dtype="bf16", n=16, t=8192, even=True, prefix=0, hq=12, hk=12, d=64, causal=False, mask=7),
        # Documents of different lengths packed in a row, grouped heads, queries and values trained (adapters on those two).
        dict(name="attend_packed_bf16", op="attend", dtype="bf16", n=7, t=8192, even=False, prefix=0, hq=32, hk=8, d=128, causal=True, mask=5),
        # Long prompts before they are answered.
        dict(name="attend_prompt_bf16", op="attend", dtype="bf16", n=2, t=16384, even=True, prefix=0, hq=32, hk=8, d=128, causal=True, mask=0),
        # float32, odd lengths and head size, keys before the first query, everything trained.
        dict(name="attend_ragged_f32", op="attend", dtype="f32", n=5, t=1777, even=False, prefix=37, hq=6, hk=2, d=72, causal=True, mask=7),
        # A token of each of 64 requests into the cache.
        dict(name="append_token_bf16", op="append", dtype="bf16", n=64, t=64, past=4000, hq=32, hk=8, d=128, r=128, pairs=False, page=16),
        # The prompts of 5 requests into the cache.
        dict(name="append_prompt_bf16", op="append", dtype="bf16", n=5, t=16384, past=0, hq=32, hk=8, d=128, r=128, pairs=False, page=64),
        # One request's next token.
        dict(name="paged_token_bf16", op="paged", dtype="bf16", n=1, keys=4111, hq=32, hk=8, d=128, page=16),
        # The next token of 64 requests with caches of different lengths.
        dict(name="paged_batch_bf16", op="paged", dtype="bf16", n=64, keys=400000, hq=32, hk=8, d=128, page=64),
        # float32, odd page and head sizes, five query heads to one of the cache.
        dict(name="paged_ragged_f32", op="paged", dtype="f32", n=9, keys=20011, hq=15, hk=3, d=100, page=24),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    """Query heads, heads of keys and values, head size: usually what models have, sometimes anything."""
    hk, group = rng.choice([1, 2, 4, 8, 8, 12, 5]), rng.choice([1, 1, 2, 4, 4, 8, 3])
    while hk * group > 40:
        group -= 1
    d = rng.choice([64, 64, 128, 128, 128, 80, 96, 256]) if rng.random() < 0.7 else rng.randint(16, 256)
    return dict(hq=hk * group, hk=hk, d=d)


def _turn(rng, d):
    """How much of a head turns, and in which pairs."""
    r = d - d % 2 if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
    return dict(r=r, pairs=rng.random() < 0.4)


def draw(rng):
    op, dtype = rng.choice(["rotary", "attend", "attend", "append", "paged", "paged"]), rng.choice(["bf16", "bf16", "f32"])
    h = _heads(rng)
    if op == "rotary":
        t = min(_log(rng, 1, 16384), 42_000_000 // ((h["hq"] + h["hk"]) * h["d"]))
        return dict(op=op, dtype=dtype, t=t, **h, **_turn(rng, h["d"]), far=_log(rng, 16, 1000000), mask=rng.choice([0, 0, 1, 6, 7]))
    if op == "attend":
        n, t = _log(rng, 1, 64), _log(rng, 16, 16384)
        c = dict(op=op, dtype=dtype, n=min(n, t), t=t, even=rng.random() < 0.3, prefix=rng.choice([0, 0, 0, rng.randint(1, 500)]), **h,
                 causal=rng.random() < 0.7, mask=rng.choice([0, 0, 1, 3, 4, 5, 7, 7]))
        # at most these many operations a pass, and elements of scores
        while (f := work(c)["flops"]) > {"bf16": 1e12, "f32": 8e10}[dtype] or f > 8e9 * h["d"]:
            c["t"] = c["t"] * 4 // 5
            c["n"] = min(n, c["t"])
        return c
    page = rng.choice([16, 16, 32, 64, 128, 24, 5])
    if op == "append":
        if rng.random() < 0.5:
            n = t = _log(rng, 1, 256)
            past = _log(rng, 1, 20000)
        else:
            t, past = min(_log(rng, 16, 16384), 60_000_000 // ((h["hq"] + 2 * h["hk"]) * h["d"])), rng.choice([0, 0, 777])
            n = min(t, _log(rng, 1, 32))
        return dict(op=op, dtype=dtype, n=n, t=t, past=min(past, 1_000_000 // n), **h, **_turn(rng, h["d"]), page=page)
    n = _log(rng, 1, 128)
    keys = min(max(n, _log(rng, 1, 400000)), 400_000_000 // (h["hk"] * h["d"] * (2 if dtype == "f32" else 1)))
    return dict(op=op, dtype=dtype, n=n, keys=max(n, keys), **h, page=page)


# ------------------------------------------------------------------ inputs
def _lengths(n, total, even):
    """n lengths of at least one with this sum, a matter of the case alone."""
    if even:
        return [total // n + (1 if i < total % n else 0) for i in range(n)]
    rng = random.Random(1000003 * n + total)
    share = [rng.random() ** 2 + 0.02 for _ in range(n)]
    out = [1 + int((total - n) * s / sum(share)) for s in share]
    out[0] += total - sum(out)
    return out


def _spans(case):
    """(first query, queries, first key, keys) of each sequence."""
    out, a, b = [], 0, 0
    for m in _lengths(case["n"], case["t"], case["even"]):
        out.append((a, m, b, m + case["prefix"]))
        a, b = a + m, b + m + case["prefix"]
    return out


def _starts(sizes):
    out = [0]
    for s in sizes:
        out.append(out[-1] + s)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hk, d = DTYPES[case["dtype"]], case["hq"], case["hk"], case["d"]

    def normal(shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dt)

    def heads(t, h):
        # projections of hidden states: a few channels of each head stand out
        x = torch.empty((t, h, d), device="cuda").normal_(0.0, 1.0, generator=g)
        x[:, :, :: max(1, d // 4)] *= 4.0
        return x.to(dt)

    s = dict(case)
    if case["op"] in ("rotary", "append"):
        r = case["r"]
        s["freq"] = torch.tensor([THETA ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float32, device="cuda")
        s.update(gq=normal(d, 0.2, 1.0), gk=normal(d, 0.2, 1.0))
    if case["op"] == "rotary":
        t = case["t"]
        s["positions"] = torch.randint(0, case["far"], (t,), dtype=torch.int32, device="cuda", generator=g)
        s.update(x=heads(t, hq + hk), gy=normal((t, hq + hk, d)))
        return s
    if case["op"] == "attend":
        spans, t = _spans(case), case["t"]
        s["offsets"] = _starts([m for _, m, _, _ in spans])
        s["k_offsets"] = _starts([m for _, _, _, m in spans]) if case["prefix"] else None
        if case["prefix"]:
            s.update(q=normal((t, hq, d), 1.5), k=normal((t + case["n"] * case["prefix"], hk, d)))
            s["v"] = normal(s["k"].shape)
        else:
            # one projection holds all three, as a Linear writes it
            p = torch.empty((t, hq + 2 * hk, d), device="cuda").normal_(0.0, 1.0, generator=g)
            p[:, :hq] *= 1.5
            p = p.to(dt)
            s.update(q=p[:, :hq], k=p[:, hq:hq + hk], v=p[:, hq + hk:])
        s["gy"] = normal((t, hq, d))
        return s
    page = case["page"]
    if case["op"] == "append":
        fresh = _lengths(case["n"], case["t"], case["t"] == case["n"])
        lengths = [case["past"] + m for m in fresh]
        s["rows"] = torch.repeat_interleave(torch.arange(case["n"], dtype=torch.int32, device="cuda"), torch.tensor(fresh, device="cuda"))
        s["positions"] = (torch.arange(case["t"], device="cuda") - _starts(fresh)[:-1].long()[s["rows"].long()] + case["past"]).to(torch.int32)
        s["x"] = heads(case["t"], hq + 2 * hk)
    else:
        lengths = _lengths(case["n"], case["keys"], False)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["q"] = normal((case["n"], hq, d), 1.5)
    # pages in no order, a few more than are used
    need = [-(-m // page) for m in lengths]
    pages, wide = sum(need) + 3, max(need)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    at = torch.arange(wide, device="cuda")[None, :] + _starts(need)[:-1].long()[:, None]
    s["tables"] = torch.where(torch.arange(wide, device="cuda")[None, :] < torch.tensor(need, device="cuda")[:, None],
                              order[at.clamp(max=pages - 1)], 0).to(torch.int32).contiguous()
    s.update(k_pages=normal((pages, hk, page, d)), v_pages=normal((pages, hk, page, d)))
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ------------------------------------------------------------------ the library's operators
def _run_own(s):
    import paper_2404_12406_amd as ms
    if s["op"] == "rotary":
        spec = ms.HeadNormRotary(s["positions"], s["freq"], q_heads=s["hq"], eps=EPS, interleaved=s["pairs"])
        y, rec = ms.layer_forward(spec, s["x"], s["gq"], s["gk"], mask=s["mask"])
    elif s["op"] == "attend":
        spec = ms.Attention(s["offsets"], s["k_offsets"], causal=s["causal"])
        y, rec = ms.layer_forward(spec, s["q"], s["k"], s["v"], mask=s["mask"])
    elif s["op"] == "append":
        spec = ms.CacheAppend(s["k_pages"], s["v_pages"], s["tables"], s["positions"], s["rows"], s["freq"], q_heads=s["hq"], eps=EPS,
                              interleaved=s["pairs"])
        y, _ = ms.layer_forward(spec, s["x"], s["gq"], s["gk"])
        return y, s["k_pages"], s["v_pages"]
    else:
        y, rec = ms.layer_forward(ms.PagedAttention(s["k_pages"], s["v_pages"], s["tables"], s["lengths"]), s["q"])
    if rec is None:
        return (y,)
    return (y,) + tuple(g for g in ms.layer_backward(rec, s["gy"]) if g is not None)


# ------------------------------------------------------------------ plain form
def _turned(z, cos, sin, pairs, back=False):
    """The first 2 len(cos) elements of each head turned by their angles, or back."""
    h = cos.shape[-1]
    if back:
        sin = -sin
    if pairs:
        a, b = z[..., 0:2 * h:2], z[..., 1:2 * h:2]
        part = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = z[..., :h], z[..., h:2 * h]
        part = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([part, z[..., 2 * h:]], -1)


def _angles(s):
    a = s["positions"].double()[:, None] * s["freq"].double()[None, :]
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _plain_rotary(s, x):
    """Normed and turned heads, what the backward needs beside them."""
    hq, h = s["hq"], s["hq"] + s["hk"]
    g = torch.cat([s["gq"].float().expand(hq, -1), s["gk"].float().expand(h - hq, -1)])
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    cos, sin = _angles(s)
    return _turned(x * r * g, cos, sin, s["pairs"]), g, r, cos, sin


def _plain_attend(s, q, k, v, gy, a, m, b, n):
    """One sequence: q, gy[Hq, m, D], k, v[Hk, n, D]."""
    hq, hk, d = s["hq"], s["hk"], s["d"]
    scale = 1.0 / math.sqrt(d)
    q, gy = q[a:a + m].transpose(0, 1).float(), gy[a:a + m].transpose(0, 1).float()
    k, v = (x[b:b + n].transpose(0, 1).float().repeat_interleave(hq // hk, 0) for x in (k, v))
    z = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
    if s["causal"]:
        i = torch.arange(n, device="cuda")
        z = z.masked_fill(i[None, :] > i[n - m:, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    del z
    o = torch.bmm(p, v)
    dq = dk = dv = None
    shared = lambda x: x.reshape(hk, hq // hk, n, d).sum(1).transpose(0, 1)  # noqa: E731
    if s["mask"] & 4:
        dv = shared(torch.bmm(p.transpose(1, 2).contiguous(), gy))
    if s["mask"] & 3:
        ds = torch.bmm(gy, v.transpose(1, 2).contiguous())
        ds = p * (ds - (gy * o).sum(-1, keepdim=True)) * scale
        if s["mask"] & 1:
            dq = torch.bmm(ds, k).transpose(0, 1)
        if s["mask"] & 2:
            dk = shared(torch.bmm(ds.transpose(1, 2).contiguous(), q))
    return o.transpose(0, 1), dq, dk, dv


def _run_plain(s):
    dt = DTYPES[s["dtype"]]
    if s["op"] == "rotary":
        x = s["x"].float()
        y, g, r, cos, sin = _plain_rotary(s, x)
        out = [y.to(dt)]
        if s["mask"]:
            dz = _turned(s["gy"].float(), cos, sin, s["pairs"], True)
            if s["mask"] & 1:
                u = dz * g
                out.append((r * (u - x * r * r * (u * x).mean(-1, keepdim=True))).to(dt))
            dg = dz * x * r
            if s["mask"] & 2:
                out.append(dg[:, :s["hq"]].sum((0, 1)).to(dt))
            if s["mask"] & 4:
                out.append(dg[:, s["hq"]:].sum((0, 1)).to(dt))
        return tuple(out)
    if s["op"] == "attend":
        parts = [_plain_attend(s, s["q"], s["k"], s["v"], s["gy"], *span) for span in _spans(s)]
        return tuple(torch.cat(p).to(dt) for p in zip(*parts) if p[0] is not None)
    page, hq, hk = s["page"], s["hq"], s["hk"]
    if s["op"] == "append":
        x = s["x"]
        y = _plain_rotary(s, x[:, :hq + hk].float())[0].to(dt)
        pos = s["positions"].long()
        at = s["tables"].long()[s["rows"].long(), pos // page]
        s["k_pages"][at, :, pos % page] = y[:, hq:]
        s["v_pages"][at, :, pos % page] = x[:, hq + hk:]
        return y[:, :hq].contiguous(), s["k_pages"], s["v_pages"]
    n, d = s["n"], s["d"]
    k, v = (p[s["tables"].long()].transpose(1, 2).reshape(n * hk, -1, d).float() for p in (s["k_pages"], s["v_pages"]))
    hidden = (torch.arange(k.shape[1], device="cuda")[None, :] >= s["lengths"][:, None]).repeat_interleave(hk, 0)[:, :, None]
    v = v.masked_fill(hidden, 0.0)
    q = s["q"].float().reshape(n * hk, hq // hk, d)
    z = torch.bmm(k, q.transpose(1, 2).contiguous()).masked_fill(hidden, -math.inf) * (1.0 / math.sqrt(d))
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    return (torch.bmm(p.transpose(1, 2).contiguous(), v).reshape(n, hq, d).to(dt),)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64 bits
def _exact_rotary(s, x):
    """x[T, Hq + Hk, D] as complex numbers of modulus and angle; differentiable."""
    g = torch.cat([s["gq64"][None].expand(s["hq"], -1), s["gk64"][None].expand(s["hk"], -1)])
    z = torch.nn.functional.normalize(x, dim=-1, eps=0.0) if EPS == 0 else x / torch.sqrt(x.square().sum(-1, keepdim=True) / s["d"] + EPS)
    z = z * g
    half = s["r"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if s["pairs"] else (i, i + half)
    w = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), s["freq"].double()))
    c = torch.complex(z[..., first], z[..., second]) * w[:, None, :]
    y = z.clone()
    y[..., first] = c.real
    y[..., second] = c.imag
    return y


def exact(case, seed):
    """The definitions in 64 bits; gradients by differentiating them."""
    s = _inputs(case, seed)
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["op"] in ("rotary", "append"):
        s["gq64"], s["gk64"] = s["gq"].double(), s["gk"].double()
    if case["op"] == "rotary":
        x = s["x"].double()
        leaves = [x, s["gq64"], s["gk64"]]
        want = [t.requires_grad_() for bit, t in zip((1, 2, 4), leaves) if case["mask"] & bit]
        y = _exact_rotary(s, x)
        return (y.detach(),) + (torch.autograd.grad(y, want, s["gy"].double()) if want else ())
    if case["op"] == "append":
        y = _exact_rotary(s, s["x"][:, :hq + hk].double())
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        pos = s["positions"].long()
        flat = s["tables"].long()[s["rows"].long(), torch.div(pos, case["page"], rounding_mode="floor")] * case["page"] + pos % case["page"]
        for pages, new in ((kp, y[:, hq:]), (vp, s["x"][:, hq + hk:].double())):
            rows = pages.transpose(1, 2).reshape(-1, hk, d)
            rows[flat] = new
            pages.copy_(rows.reshape(pages.shape[0], case["page"], hk, d).transpose(1, 2))
        return y[:, :hq], kp, vp
    scale = d ** -0.5
    if case["op"] == "paged":
        out = torch.empty((case["n"], hq, d), dtype=torch.float64, device="cuda")
        for b, m in enumerate(s["lengths"].tolist()):
            used = s["tables"][b, :-(-m // case["page"])].long()
            k, v = (p[used].double().permute(1, 0, 2, 3).flatten(1, 2)[:, :m] for p in (s["k_pages"], s["v_pages"]))
            q = s["q"][b].double().reshape(hk, hq // hk, d)
            out[b] = (torch.softmax(q @ k.mT * scale, -1) @ v).reshape(hq, d)
        return (out,)
    outs = [torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in ("q", "q", "k", "v")]
    for a, m, b, n in _spans(case):
        for h in range(hq):
            c = h * hk // hq
            leaves = [s["q"][a:a + m, h].double(), s["k"][b:b + n, c].double(), s["v"][b:b + n, c].double()]
            want = [t.requires_grad_() for bit, t in zip((1, 2, 4), leaves) if case["mask"] & bit]
            z = (leaves[0] @ leaves[1].mT) * scale
            if case["causal"]:
                z = z.masked_fill(torch.ones(m, n, dtype=torch.bool, device="cuda").triu(n - m + 1), -math.inf)
            o = torch.softmax(z, -1) @ leaves[2]
            outs[0][a:a + m, h] = o.detach()
            if want:
                grads = iter(torch.autograd.grad(o, want, s["gy"][a:a + m, h].double()))
                for bit, to, head in ((1, outs[1], h), (2, outs[2], c), (4, outs[3], c)):
                    if case["mask"] & bit:
                        to[(a if bit == 1 else b):(a + m if bit == 1 else b + n), head] += next(grads)
    return (outs[0],) + tuple(t for bit, t in zip((1, 2, 4), outs[1:]) if case["mask"] & bit)


# ------------------------------------------------------------------ work
def work(case):
    """Inputs read once, outputs written once; of attention the products over the pairs that are
    visible, backward the scores once more, the gradient of the probabilities where q or k asks for
    it, and one for each gradient."""
    e, hq, hk, d = ELT[case["dtype"]], case["hq"], case["hk"], case["d"]
    if case["op"] == "rotary":
        n, mask = case["t"] * (hq + hk) * d, case["mask"]
        b = 2 * n + 2 * d
        if mask:
            b += n + (n if mask & 1 else 0) + (d if mask & 2 else 0) + (d if mask & 4 else 0)
        return {"bytes": b * e + 4 * case["t"] + 2 * case["r"], "flops": 7 * n + (13 * n if mask else 0)}
    if case["op"] == "append":
        n = case["t"] * (hq + 2 * hk) * d
        return {"bytes": 2 * n * e + 12 * case["t"] + 2 * case["r"], "flops": 7 * n}
    if case["op"] == "paged":
        pages = sum(-(-m // case["page"]) for m in _lengths(case["n"], case["keys"], False))
        return {"bytes": (2 * case["keys"] * hk * d + 2 * case["n"] * hq * d) * e + 4 * (pages + case["n"]), "flops": 4 * case["keys"] * hq * d}
    pairs = keys = 0
    for _, m, _, n in _spans(case):
        pairs += m * n - (m * (m - 1) // 2 if case["causal"] else 0)
        keys += n
    nq, nk, mask = case["t"] * hq * d, keys * hk * d, case["mask"]
    b, products = 2 * nq + 2 * nk, 2
    if mask:
        b += nq + (nq if mask & 1 else 0) + (nk if mask & 2 else 0) + (nk if mask & 4 else 0)
        products += 1 + (1 if mask & 3 else 0) + (mask & 1) + (mask >> 1 & 1) + (mask >> 2 & 1)
    return {"bytes": b * e, "flops": 2 * pairs * hq * d * products}
