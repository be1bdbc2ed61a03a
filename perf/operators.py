"""The transformer layers of this library -- layer norm, gated linear unit and
linear cross entropy -- as measurable cases.

One pass is one layer as a program calls it: the forward alone where nothing
asks for a gradient (serving, scoring), else the forward and the backward
that writes exactly the gradients the mask asks for.  The plain form is the
same mathematics in elementary torch operations, in 32 bits, rounded once at
the end; `exact` is the definition again in 64 bits.

    layer norm      y = (x - mean) / sqrt(var + eps) * gamma + beta over rows of x[M, D]
    gated linear    y = act(x Wg^T + bg) * (x Wu^T + bu), W = [Wg; Wu][2F, D], b = [bg; bu]
    cross entropy   loss = mean (or sum, or each) over the rows i whose target t is not ignored of
                    log sum_v exp(z_iv) - z_it, z = x W^T + b, x[M, D], W[V, D]
"""
import math

import torch

own = False   # plain form (False) or the library's kernels (True)

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ELT = {"f32": 4, "bf16": 2}
EPS = 1e-5
IGNORE = -100


def listed():
    return [
        # One token through a norm while a model answers: launch latency is all of it.
        dict(name="norm_token_bf16", op="norm", dtype="bf16", m=1, d=768, mask=0),
        # The norm of an encoder layer on 16 x 512 tokens, scale and shift trained.
        dict(name="norm_train_bf16", op="norm", dtype="bf16", m=8192, d=768, mask=7),
        # Rows that no vector width divides, float32, everything trained.
        dict(name="norm_ragged_f32", op="norm", dtype="f32", m=3001, d=2051, mask=7),
        # Wide rows, affine frozen: fine-tuning below an adapter.
        dict(name="norm_wide_bf16", op="norm", dtype="bf16", m=16384, d=4096, mask=1),
        # One token through the gated half of a feed-forward block: the weights are read once.
        dict(name="gated_token_bf16", op="gated", dtype="bf16", m=1, d=4096, f=10944, act="silu", keep="projections",
             bias=False, mask=0),
        # The encoder's hidden size and tokens with a gated block of the same
        # parameters as its 4-fold one (2/3 as wide), trained.
        dict(name="gated_train_bf16", op="gated", dtype="bf16", m=8192, d=768, f=2048, act="gelu", keep="projections",
             bias=True, mask=7),
        # A larger block with its weights frozen, keeping its input alone.
        dict(name="gated_frozen_bf16", op="gated", dtype="bf16", m=4096, d=2048, f=5504, act="silu", keep="input",
             bias=False, mask=1),
        # float32, odd rows and widths, trained.
        dict(name="gated_ragged_f32", op="gated", dtype="f32", m=1001, d=515, f=1366, act="gelu_tanh",
             keep="projections", bias=True, mask=7),
        # Log-probability of the next token of four requests under a language model's head.
        dict(name="xent_score_bf16", op="xent", dtype="bf16", m=4, d=768, v=50000, bias=False, ignored=0.0,
             reduction="none", mask=0),
        # A trained head on 16 x 512 tokens, a third of them a prompt that does not count.
        dict(name="xent_train_bf16", op="xent", dtype="bf16", m=8192, d=768, v=50000, bias=False, ignored=0.34,
             reduction="mean", mask=3),
        # A large vocabulary, the head frozen: gradients to the hidden states alone.
        dict(name="xent_frozen_bf16", op="xent", dtype="bf16", m=4096, d=4096, v=128000, bias=False, ignored=0.0,
             reduction="mean", mask=1),
        # A float32 classifier over an odd number of words, with a bias, trained.
        dict(name="xent_ragged_f32", op="xent", dtype="f32", m=777, d=514, v=10007, bias=True, ignored=0.1,
             reduction="sum", mask=7),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer width: usually what models have, sometimes anything."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.3:
        return n
    step = 64 if n < 2048 else 128
    return min(hi, max(step, n // step * step))


def draw(rng):
    op, dtype = rng.choice(["norm", "gated", "gated", "xent", "xent"]), rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        m, d = _log(rng, 1, 16384), _width(rng, 64, 8192)
        return dict(op=op, dtype=dtype, m=max(1, min(m, 16384 * 4096 // d)), d=d, mask=rng.choice([0, 1, 6, 7]))
    # products of at most these many multiply-adds a pass forward, by type
    most = 92e9 if dtype == "bf16" else 12e9
    few = rng.random() < 0.3
    m = rng.randint(1, 16) if few else _log(rng, 17, 8192)
    mask = 0 if few else rng.choice([0, 1, 3, 7, 7])
    bias = mask & 4 != 0 or rng.random() < 0.3
    d = _width(rng, 128, 4096)
    if op == "gated":
        f = _width(rng, 128, 10944)
        return dict(op=op, dtype=dtype, m=max(1, min(m, int(most / (2 * d * f)))), d=d, f=f,
                    act=rng.choice(["silu", "gelu", "gelu_tanh", "sigmoid"]), keep=rng.choice(["projections", "input"]),
                    bias=bias, mask=mask)
    # the head and its gradient in at most a gigabyte
    v = min(_log(rng, 1000, 128000), int(1e9 / (ELT[dtype] * d * (2 if mask & 2 else 1))))
    return dict(op=op, dtype=dtype, m=max(1, min(m, int(most / (d * v)))), d=d, v=v, bias=bias,
                ignored=rng.choice([0.0, 0.0, 0.3, 0.9]), reduction=rng.choice(["mean", "sum", "none"]), mask=mask)


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, m, d = DTYPES[case["dtype"]], case["m"], case["d"]

    def normal(shape, std=1.0, mean=0.0):
        t = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g)
        return t.to(dt)

    s = dict(case)
    if case["op"] == "norm":
        # hidden states have a few channels that stand out
        x = torch.empty((m, d), device="cuda").normal_(0.3, 1.0, generator=g)
        x[:, :: max(1, d // 8)] *= 6.0
        s.update(x=x.to(dt), W=normal(d, 0.2, 1.0), b=normal(d, 0.1), gy=normal((m, d)))
    elif case["op"] == "gated":
        f = case["f"]
        s.update(x=normal((m, d)), W=normal((2 * f, d), 1.0 / math.sqrt(d)), b=normal(2 * f, 0.1) if case["bias"] else None,
                 gy=normal((m, f)))
    else:
        v = case["v"]
        W = torch.empty((v, d), device="cuda").normal_(0.0, 0.02, generator=g)
        t = torch.randint(0, v, (m,), device="cuda", generator=g)
        # a model that has learned something: the target's logit stands some 5 above the others'
        x = torch.empty((m, d), device="cuda").normal_(0.0, 1.0, generator=g) + W[t] * (5.0 / (4e-4 * d))
        drop = torch.rand((m,), device="cuda", generator=g) < case["ignored"]
        if case["reduction"] == "mean":
            drop[0] = False   # a mean over no row has no value
        rows = m if case["reduction"] == "none" else 1
        s.update(x=x.to(dt), W=W.to(dt), b=normal(v, 0.1) if case["bias"] else None, target=torch.where(drop, IGNORE, t),
                 gy=torch.empty(rows, device="cuda").uniform_(0.5, 1.5, generator=g))
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ------------------------------------------------------------------ the library's layers
def _run_own(s):
    import paper_2404_12406_amd as ms
    if s["op"] == "norm":
        spec = ms.LayerNorm(EPS)
    elif s["op"] == "gated":
        spec = ms.GatedLinear(s["act"], keep=s["keep"])
    else:
        spec = ms.LinearCrossEntropy(s["target"], ignore_index=IGNORE, reduction=s["reduction"])
    y, rec = ms.layer_forward(spec, s["x"], s["W"], s["b"], mask=s["mask"])
    if rec is None:
        return (y,)
    grads = ms.layer_backward(rec, s["gy"])
    return (y,) + tuple(g for g in grads if g is not None)


# ------------------------------------------------------------------ plain form
def _grads(mask, dx, dW, db):
    out = []
    for bit, g in ((1, dx), (2, dW), (4, db)):
        if mask & bit:
            out.append(g())
    return out


def _act(name, g):
    """act(g) and its derivative."""
    if name == "sigmoid":
        a = 1.0 / (1.0 + torch.exp(-g))
        return a, a * (1.0 - a)
    if name == "silu":
        a = 1.0 / (1.0 + torch.exp(-g))
        return g * a, a * (1.0 + g * (1.0 - a))
    if name == "gelu":
        c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * g * g)


def _run_plain(s):
    dt, mask = s["x"].dtype, s["mask"]
    x, W, b = (None if s[k] is None else s[k].float() for k in ("x", "W", "b"))
    gy = s["gy"].float()
    if s["op"] == "norm":
        c = x - x.mean(1, keepdim=True)
        r = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
        h = c * r
        out = [h * W + b]
        if mask:
            def dx():
                q = gy * W
                return r * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
            out += _grads(mask, dx, lambda: (gy * h).sum(0), lambda: gy.sum(0))
        return tuple(o.to(dt) for o in out)
    z = x @ W.t()
    if b is not None:
        z = z + b
    if s["op"] == "gated":
        f = s["f"]
        g, u = z[:, :f], z[:, f:]
        a, da = _act(s["act"], g)
        out = [a * u]
        if mask:
            dz = torch.cat([gy * u * da, gy * a], 1)
            out += _grads(mask, lambda: dz @ W, lambda: dz.t() @ x, lambda: dz.sum(0))
        return tuple(o.to(dt) for o in out)
    t = s["target"]
    counts = t != IGNORE
    tc = torch.where(counts, t, 0)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    each = torch.where(counts, (top + torch.log(total) - z.gather(1, tc[:, None]))[:, 0], 0.0)
    n = counts.sum()
    loss = each if s["reduction"] == "none" else each.sum().reshape(1) / (n if s["reduction"] == "mean" else 1)
    out = []
    if mask:
        scale = torch.where(counts, gy / n if s["reduction"] == "mean" else gy, 0.0)
        dz = e / total
        dz.scatter_add_(1, tc[:, None], torch.full_like(dz[:, :1], -1.0))
        dz *= scale[:, None]
        out = _grads(mask, lambda: dz @ W, lambda: dz.t() @ x, lambda: dz.sum(0))
    return (loss,) + tuple(o.to(dt) for o in out)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64 bits
def _act64(name, g):
    if name in ("sigmoid", "silu"):
        s = torch.special.expit(g)
        ds = s * torch.special.expit(-g)
        return (s, ds) if name == "sigmoid" else (g * s, s + g * ds)
    if name == "gelu":
        phi = torch.exp(g.square() / -2) / math.sqrt(2 * math.pi)
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * phi
    # 0.5 (1 + tanh(p)) = 1 / (1 + exp(-2 p))
    p2 = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    s = torch.special.expit(p2)
    return g * s, s + g * s * (1 - s) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)


def exact(case, seed):
    """The definitions in 64 bits, some rows at a time."""
    s = _inputs(case, seed)
    mask, m, d = case["mask"], case["m"], case["d"]
    x, W, gy = s["x"].double(), s["W"].double(), s["gy"].double()
    b = None if s["b"] is None else s["b"].double()
    if case["op"] == "norm":
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        sd = torch.sqrt(var + EPS)
        h = (x - mean) / sd
        out = [torch.addcmul(b, h, W)]
        if mask & 1:
            q = gy * W
            out.append((d * q - q.sum(1, keepdim=True) - h * torch.linalg.vecdot(q, h).unsqueeze(1)) / (d * sd))
        if mask & 2:
            out.append(torch.einsum("md,md->d", gy, h))
        if mask & 4:
            out.append(torch.ones(m, dtype=torch.float64, device="cuda") @ gy)
        return tuple(out)
    gated = case["op"] == "gated"
    rows = max(1, int(2e8) // W.shape[0])
    ys, dxs = [], []
    dW = torch.zeros_like(W) if mask & 2 else None
    db = torch.zeros(W.shape[0], dtype=torch.float64, device="cuda") if mask & 4 else None
    live = None if gated else s["target"] != IGNORE
    share = 1.0
    if not gated and case["reduction"] == "mean":
        share = 1.0 / int(live.sum())
    for i in range(0, m, rows):
        xi = x[i:i + rows]
        z = torch.addmm(b, xi, W.t()) if b is not None else torch.mm(xi, W.t())
        if gated:
            f, gi = case["f"], gy[i:i + rows]
            a, da = _act64(case["act"], z[:, :f])
            ys.append(a * z[:, f:])
            if mask:
                dz = torch.empty_like(z)
                dz[:, :f] = da * z[:, f:] * gi
                dz[:, f:] = a * gi
        else:
            li = live[i:i + rows]
            ti = torch.where(li, s["target"][i:i + rows], 0)
            lse = torch.logsumexp(z, 1)
            pick = torch.arange(len(ti), device="cuda")
            ys.append(torch.where(li, lse - z[pick, ti], 0.0))
            if mask:
                dz = torch.exp(z - lse[:, None])
                dz[pick, ti] -= 1.0
                w = (gy[i:i + rows] if case["reduction"] == "none" else gy.expand(len(ti))) * share
                dz *= torch.where(li, w, 0.0)[:, None]
        if mask & 1:
            dxs.append(dz @ W)
        if mask & 2:
            dW += dz.t() @ xi
        if mask & 4:
            db += dz.sum(0)
    y = torch.cat(ys)
    if not gated and case["reduction"] != "none":
        y = (y.sum() * share).reshape(1)
    out = [y]
    if mask & 1:
        out.append(torch.cat(dxs))
    if mask & 2:
        out.append(dW)
    if mask & 4:
        out.append(db)
    return tuple(out)


# ------------------------------------------------------------------ work
def work(case):
    """Inputs read once, outputs written once, and the products (of rows that
    count) with the gradients' ones where the mask asks for them."""
    e, m, d, mask = ELT[case["dtype"]], case["m"], case["d"], case["mask"]
    if case["op"] == "norm":
        n, p = m * d, 2 * d
        b = 2 * n + p
        if mask:
            b += n + (n if mask & 1 else 0) + (d if mask & 2 else 0) + (d if mask & 4 else 0)
        return {"bytes": b * e, "flops": 8 * n + (10 * n if mask else 0)}
    out = 2 * case["f"] if case["op"] == "gated" else case["v"]
    w = out * d
    b = (m * d + w + (out if case["bias"] else 0)) * e
    b += m * case["f"] * e if case["op"] == "gated" else 8 * m + 4 * (m if case["reduction"] == "none" else 1)
    live = 1.0 if case["op"] == "gated" else 1.0 - case["ignored"]
    fl = 2.0 * m * live * w
    total = fl
    if mask:
        b += m * case["f"] * e if case["op"] == "gated" else 4 * (m if case["reduction"] == "none" else 1)
        b += (m * d if mask & 1 else 0) * e + (w if mask & 2 else 0) * e + (out if mask & 4 else 0) * e
        total += fl * ((mask & 1) + (mask >> 1 & 1))
    return {"bytes": int(b), "flops": int(total)}
