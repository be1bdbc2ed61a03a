"""Attention's entry points without a GPU (attention.cpp with stub launchers): what they
refuse, what their records borrow by mask, the ledger, tensors in other layouts, a workspace
that cannot be had."""
import ctypes
import os
import subprocess

import pytest

from paper_2404_12406_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NATIVE = os.path.join(ROOT, "tests", "native")
BUILD = os.path.join(NATIVE, "_build")
FAKE = 0x7f0000000000   # an aligned address that nobody reads
OUT = FAKE + (1 << 40)  # another, of results
DT = {"f32": L.MS_F32, "bf16": L.MS_BF16}
SAVED_X, SAVED_W, SAVED_Y, SAVED_LSE, SAVED_B, SAVED_INDEX = 1, 2, 32, 256, 1024, 2048


@pytest.fixture(scope="module")
def stub():
    os.makedirs(BUILD, exist_ok=True)
    so = os.path.join(BUILD, "libmemsave_attention.so")
    csrc = os.path.join(ROOT, "paper_2404_12406_amd", "csrc")
    tmp = so + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", os.path.join(ROOT, "include")]
                   + [os.path.join(csrc, f) for f in ("memsave.cpp", "blocks.cpp", "attention.cpp")]
                   + [os.path.join(NATIVE, f) for f in ("host_stub.cpp", "blocks_stub.cpp", "attention_stub.cpp")] + ["-o", tmp],
                   check=True)
    os.replace(tmp, so)
    lib = L.configure(ctypes.CDLL(so))
    for f in ("attention_log", "attention_violations", "stub_log"):
        getattr(lib, f).restype = ctypes.c_char_p
    lib.attention_reset()
    lib.stub_reset()
    return lib


@pytest.fixture(autouse=True)
def clean(stub):
    live0 = live(stub)
    yield
    assert stub.attention_violations() == b""
    assert live(stub) == live0
    reset(stub)


def reset(lib):
    lib.attention_reset()
    lib.stub_reset()


def live(lib):
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    lib.ms_ledger_read(ctypes.byref(a), ctypes.byref(b))
    return a.value


def tensor(shape, dtype="bf16", strides=None, addr=FAKE):
    t = L.MsTensor()
    t.data, t.dtype, t.ndim = addr, DT.get(dtype, dtype), len(shape)
    if strides is None:
        strides, n = [], 1
        for s in reversed(shape):
            strides.insert(0, n)
            n *= max(s, 1)
    for i, (s, st) in enumerate(zip(shape, strides)):
        t.shape[i], t.stride[i] = s, st
    return t


def ref(t):
    return ctypes.byref(t) if t is not None else None


TQ, TK, HQ, HK, D, PAGES, PAGE, WIDTH = 12, 20, 6, 2, 40, 9, 8, 3


class Call:
    """One forward with its good arguments, any of which a test replaces."""

    def __init__(self, lib, kind, dtype="bf16", **over):
        self.lib, self.kind, self.dtype = lib, kind, dtype
        self.a = a = dict(mask=7, rec=True, eps=1e-6, qh=HQ, R=D, next=0, norm=1, pos=FAKE, freq=FAKE, rotary=True, scale=0.25, causal=1,
                          gq=tensor((D,), dtype), gk=tensor((D,), dtype), tables=FAKE, n=TQ, width=WIDTH,
                          kp=tensor((PAGES, HK, PAGE, D), dtype), vp=tensor((PAGES, HK, PAGE, D), dtype))
        if kind == "rotary":
            a.update(x=tensor((TQ, HQ + HK, D), dtype), y=tensor((TQ, HQ + HK, D), dtype, addr=OUT))
        elif kind == "attention":
            a.update(x=tensor((TQ, HQ, D), dtype), gq=tensor((TK, HK, D), dtype), gk=tensor((TK, HK, D), dtype), y=tensor((TQ, HQ, D), dtype, addr=OUT),
                     qoff=FAKE, koff=FAKE, n=3, kept=FAKE)
        elif kind == "append":
            a.update(x=tensor((TQ, HQ + 2 * HK, D), dtype), y=tensor((TQ, HQ, D), dtype, addr=OUT), rows=None, mask=0)
        else:
            a.update(x=tensor((TQ, HQ, D), dtype), y=tensor((TQ, HQ, D), dtype, addr=OUT), lengths=FAKE, mask=0)
        a.update(over)
        self.h = ctypes.c_void_p()

    def forward(self):
        a, lib = self.a, self.lib
        hp = ctypes.byref(self.h) if a["rec"] else None
        rot = ctypes.byref(L.MsRotary(a["qh"], a["R"], a["next"], a["norm"], a["eps"], a["pos"], a["freq"])) if a["rotary"] else None
        x, gq, gk, y, kp, vp = (ref(a[n]) for n in ("x", "gq", "gk", "y", "kp", "vp"))
        if self.kind == "rotary":
            return lib.ms_head_norm_rotary_forward(x, gq, gk, rot, a["mask"], y, hp, None)
        if self.kind == "attention":
            return lib.ms_attention_forward(x, gq, gk, a["qoff"], a["koff"], a["n"], a["causal"], a["scale"], a["kept"], a["mask"], y, hp, None)
        if self.kind == "append":
            return lib.ms_cache_append(x, gq, gk, rot, kp, vp, a["tables"], a["n"], a["width"], a["rows"], y, None)
        return lib.ms_paged_attention_forward(x, kp, vp, a["tables"], a["n"], a["width"], a["lengths"], a["scale"], y, None)

    def backward(self, dy="default", entry="ms_layer_backward", mask=None):
        a, m = self.a, self.a["mask"] if mask is None else mask
        if dy == "default":
            dy = a["y"]
        return getattr(self.lib, entry)(self.h, ref(dy), ref(a["x"]) if m & 1 else None, ref(a["gq"]) if m & 2 else None,
                                        ref(a["gk"]) if m & 4 else None, None)

    def account(self):
        acct = L.MsAccount()
        assert self.lib.ms_record_account(self.h, ctypes.byref(acct)) == 0
        return acct

    def free(self):
        self.lib.ms_record_free(self.h)


KINDS = ["rotary", "attention", "append", "paged"]
TRAINED = ["rotary", "attention"]


@pytest.mark.parametrize("mask,norm", [(m, 1) for m in range(8)] + [(0, 0), (1, 0)])   # (without a norm there are no scales)
@pytest.mark.parametrize("R", [0, 16])
def test_rotary_records_borrow_what_the_mask_needs(stub, mask, norm, R):
    c = Call(stub, "rotary", mask=mask, R=R, norm=norm, **({} if norm else dict(gq=None, gk=None)))
    before = live(stub)
    assert c.forward() == 0 and stub.attention_log() == b"rotary;"
    if not mask:
        assert not c.h.value and live(stub) == before
        return
    acct = c.account()
    scales = norm and mask & 1   # a scale is a factor of dx alone
    kept = (TQ * (HQ + HK) * D * 2 if norm else 0) + (TQ * 4 if R else 0)
    want = (SAVED_X if norm else 0) | (SAVED_W | SAVED_B if scales else 0) | (SAVED_INDEX if R else 0)
    assert (acct.borrowed, acct.saved_activation_bytes, acct.referenced_param_bytes) == (want, kept, (2 * D * 2 if scales else 0) + R // 2 * 4)
    assert live(stub) == before + kept
    reset(stub)
    assert c.backward() == 0
    grads = ("+dx" if mask & 1 else "") + ("+dgq" if mask & 2 else "") + ("+dgk" if mask & 4 else "")
    assert stub.attention_log().decode() == f"rotary_bwd{grads};"
    assert c.backward() == L.MS_E_CONSUMED
    c.free()


@pytest.mark.parametrize("packed", [0, 1, 2])
@pytest.mark.parametrize("mask", range(8))
def test_attention_records_borrow_what_the_mask_needs(stub, mask, packed):
    c = Call(stub, "attention", mask=mask, kept=FAKE if mask else None, qoff=FAKE if packed else None, koff=FAKE if packed == 2 else None)
    before = live(stub)
    assert c.forward() == 0
    assert stub.attention_log() == (b"attention+lse;" if mask else b"attention;")
    if not mask:
        assert not c.h.value and live(stub) == before
        return
    acct = c.account()
    both = mask & 3   # dP = dO v^T is in dq and dk alone, and so is the sum over o
    want = SAVED_X | SAVED_W | SAVED_LSE | (SAVED_B | SAVED_Y if both else 0) | (SAVED_INDEX if packed else 0)
    kept = TQ * HQ * D * 2 + TK * HK * D * 2 + TQ * HQ * 4 + (TK * HK * D * 2 + TQ * HQ * D * 2 if both else 0) + 4 * 4 * packed
    assert (acct.borrowed, acct.saved_activation_bytes, acct.referenced_param_bytes) == (want, kept, 0)
    assert live(stub) == before + kept
    reset(stub)
    assert c.backward() == 0
    grads = ("+dq" if mask & 1 else "") + ("+dk" if mask & 2 else "") + ("+dv" if mask & 4 else "")
    assert stub.attention_log().decode() == f"attention_bwd{grads};"
    assert c.backward() == L.MS_E_CONSUMED
    c.free()


@pytest.mark.parametrize("rows,heads,mask,want", [(0, 5, 7, 0), (3, 0, 1, 0), (12, 24, 0, 0), (12, 24, 4, 12 * 24 * 4), (-1, 4, 1, 0),
                                                  (2 ** 31, 2 ** 15, 1, 2 ** 48)])
def test_kept_bytes(stub, rows, heads, mask, want):
    assert stub.ms_attention_kept_bytes(rows, heads, mask) == want


def heads(T=TQ, H=HQ, D_=D, dtype="bf16", **kw):
    return tensor((T, H, D_), dtype, **kw)


def out(*a, **kw):
    return heads(*a, addr=OUT, **kw)


def pages(*shape, dtype="bf16", **kw):
    return tensor(shape or (PAGES, HK, PAGE, D), dtype, **kw)


COMMON = [
    (L.MS_E_NULL, dict(x=None)),
    (L.MS_E_NULL, dict(x=heads(H=10, addr=None))),
    (L.MS_E_NULL, dict(y=None)),
    (L.MS_E_SHAPE, dict(x=tensor((TQ, HQ * D)))),
    (L.MS_E_SHAPE, dict(x=heads(T=-1))),
    (L.MS_E_DTYPE, dict(x=tensor((TQ, HQ, D), 9))),
    (L.MS_E_DTYPE, dict(y=out(dtype="f32"))),
    (L.MS_E_LAYOUT, dict(x=heads(strides=(-HQ * D, D, 1)))),
    (L.MS_E_LAYOUT, dict(y=out(strides=(D, D, 1)))),
]
ROTARY = [
    (L.MS_E_NULL, dict(rotary=False)), (L.MS_E_NULL, dict(pos=None)), (L.MS_E_NULL, dict(freq=None)),
    (L.MS_E_ARG, dict(pos=FAKE + 2)), (L.MS_E_ARG, dict(freq=FAKE + 1)),
    (L.MS_E_ARG, dict(R=D + 2)), (L.MS_E_ARG, dict(R=7)), (L.MS_E_ARG, dict(R=-2)),
    (L.MS_E_ARG, dict(eps=-1e-6)), (L.MS_E_ARG, dict(eps=float("nan"))), (L.MS_E_ARG, dict(eps=float("inf"))),
    (L.MS_E_ARG, dict(norm=0, mask=0)),   # scales without a norm
    (L.MS_E_SHAPE, dict(qh=-1)), (L.MS_E_SHAPE, dict(qh=HQ + 2 * HK + 1)),
    (L.MS_E_SHAPE, dict(gq=tensor((D + 1,)))), (L.MS_E_SHAPE, dict(gk=tensor((1, D)))),
    (L.MS_E_DTYPE, dict(gk=tensor((D,), "f32"))), (L.MS_E_LAYOUT, dict(gq=tensor((D,), strides=(2,)))),
]
CACHE = [
    (L.MS_E_NULL, dict(kp=None)), (L.MS_E_NULL, dict(vp=pages(addr=None))), (L.MS_E_NULL, dict(tables=None)),
    (L.MS_E_ARG, dict(tables=FAKE + 2)), (L.MS_E_SHAPE, dict(n=-1)), (L.MS_E_SHAPE, dict(width=-1)),
    (L.MS_E_SHAPE, dict(kp=tensor((PAGES, HK, PAGE * D)))), (L.MS_E_SHAPE, dict(vp=pages(PAGES + 1, HK, PAGE, D))),
    (L.MS_E_SHAPE, dict(kp=pages(PAGES, 0, PAGE, D), vp=pages(PAGES, 0, PAGE, D))),
    (L.MS_E_SHAPE, dict(kp=pages(PAGES, HK, 0, D), vp=pages(PAGES, HK, 0, D))),
    (L.MS_E_SHAPE, dict(kp=pages(-1, HK, PAGE, D))),
    (L.MS_E_SHAPE, dict(kp=pages(PAGES, HK, PAGE, D + 8), vp=pages(PAGES, HK, PAGE, D + 8))),
    (L.MS_E_DTYPE, dict(kp=pages(dtype="f32"))), (L.MS_E_LAYOUT, dict(vp=pages(strides=(HK * PAGE * D, D, HK * D, 1)))),
    (L.MS_E_UNSUPPORTED, dict(kp=pages(2 ** 29, HK, PAGE // 2, D), vp=pages(2 ** 29, HK, PAGE // 2, D))),
]
K = lambda **kw: dict(gq=heads(**{"T": TK, "H": HK, **kw}), gk=heads(**{"T": TK, "H": HK, **kw}))
REFUSED = [(k, s, o) for k in KINDS for s, o in COMMON] + [
    (k, L.MS_E_NULL, dict(rec=False)) for k in TRAINED] + [(k, L.MS_E_MASK, dict(mask=8)) for k in TRAINED] + [
    (k, s, o) for k in ("rotary", "append") for s, o in ROTARY] + [(k, s, o) for k in ("append", "paged") for s, o in CACHE] + [
    ("rotary", L.MS_E_MASK, dict(gq=None)), ("rotary", L.MS_E_MASK, dict(gk=None)),
    ("rotary", L.MS_E_SHAPE, dict(y=out(H=HQ + HK, T=TQ + 1))),
    ("rotary", L.MS_E_ARG, dict(y=heads(H=HQ + HK))),   # in place, and the backward reads x
    ("rotary", L.MS_E_UNSUPPORTED, dict(x=heads(H=HQ + HK, D_=257), y=out(H=HQ + HK, D_=257), gq=None, gk=None, mask=1)),
    ("rotary", L.MS_E_UNSUPPORTED, dict(x=heads(H=HQ + HK, D_=0), y=out(H=HQ + HK, D_=0), gq=None, gk=None, mask=1)),
    ("rotary", L.MS_E_UNSUPPORTED, dict(x=heads(T=2 ** 24, H=8, D_=16))),
    ("attention", L.MS_E_NULL, dict(gq=None)), ("attention", L.MS_E_NULL, dict(gk=None)), ("attention", L.MS_E_NULL, dict(kept=None)),
    ("attention", L.MS_E_NULL, dict(qoff=None)),   # k_offsets alone
    ("attention", L.MS_E_ARG, dict(kept=FAKE + 2)), ("attention", L.MS_E_ARG, dict(qoff=FAKE + 2)), ("attention", L.MS_E_ARG, dict(koff=FAKE + 1)),
    ("attention", L.MS_E_ARG, dict(n=-1)), ("attention", L.MS_E_ARG, dict(scale=0.0)), ("attention", L.MS_E_ARG, dict(scale=-1.0)),
    ("attention", L.MS_E_ARG, dict(scale=float("nan"))), ("attention", L.MS_E_ARG, dict(scale=float("inf"))),
    ("attention", L.MS_E_SHAPE, K(H=4)), ("attention", L.MS_E_SHAPE, K(H=0)), ("attention", L.MS_E_SHAPE, K(D_=D + 8)),
    ("attention", L.MS_E_SHAPE, dict(gk=heads(T=TK + 1, H=HK))), ("attention", L.MS_E_SHAPE, dict(y=out(T=TQ + 1))),
    ("attention", L.MS_E_DTYPE, K(dtype="f32")), ("attention", L.MS_E_LAYOUT, dict(gk=heads(T=TK, H=HK, strides=(HK * D, -D, 1)))),
    ("attention", L.MS_E_UNSUPPORTED, dict(x=heads(D_=257), y=out(D_=257), **K(D_=257))),
    ("attention", L.MS_E_UNSUPPORTED, dict(x=heads(T=1, H=65536, D_=8), y=out(T=1, H=65536, D_=8), **K(H=1, D_=8))),
    ("attention", L.MS_E_UNSUPPORTED, dict(x=heads(T=2 ** 28, H=7, D_=1), y=out(T=2 ** 28, H=7, D_=1), **K(H=1, D_=1))),
    ("attention", L.MS_E_UNSUPPORTED, dict(n=2 ** 22)),   # blocks of 128 rows
    ("append", L.MS_E_SHAPE, dict(x=heads(H=HQ + 2 * HK + 1))), ("append", L.MS_E_SHAPE, dict(y=out(H=HQ + 1))),
    ("append", L.MS_E_SHAPE, dict(n=TQ - 1)), ("append", L.MS_E_ARG, dict(rows=FAKE + 2)), ("append", L.MS_E_NULL, dict(R=0, pos=None)),
    ("paged", L.MS_E_SHAPE, dict(n=TQ + 1)), ("paged", L.MS_E_NULL, dict(lengths=None)), ("paged", L.MS_E_ARG, dict(lengths=FAKE + 2)),
    ("paged", L.MS_E_ARG, dict(scale=0.0)), ("paged", L.MS_E_ARG, dict(scale=float("nan"))), ("paged", L.MS_E_SHAPE, dict(y=out(D_=8))),
    ("paged", L.MS_E_SHAPE, dict(x=heads(H=5), y=out(H=5))), ("paged", L.MS_E_SHAPE, dict(x=heads(H=0), y=out(H=0))),
    ("paged", L.MS_E_UNSUPPORTED, dict(width=2 ** 28)), ("paged", L.MS_E_UNSUPPORTED, dict(width=2 ** 28 - 512)),
    # results where other blocks, or the backward, read
    ("attention", L.MS_E_ARG, dict(y=heads())), ("attention", L.MS_E_ARG, dict(y=heads(), x=heads(addr=FAKE + 4096), mask=0)),
    ("rotary", L.MS_E_ARG, dict(mask=0, y=heads(H=HQ + HK, strides=(D, TQ * D, 1)))), ("append", L.MS_E_ARG, dict(y=heads())),
    ("paged", L.MS_E_ARG, dict(y=heads(strides=(D, TQ * D, 1)))),
]


def name(v):
    return v if isinstance(v, str) else "+".join(v) if isinstance(v, dict) else str(v)


@pytest.mark.parametrize("kind,status,over", REFUSED, ids=name)
def test_refusals_launch_nothing(stub, kind, status, over):
    c = Call(stub, kind, **over)
    assert c.forward() == status, stub.ms_last_error()
    assert not c.h.value and stub.attention_log() == b"" and stub.stub_log() == b""


def test_generic_entry_points_refuse_these_layers(stub):
    layer, h = L.MsLayer(), ctypes.c_void_p()
    for kind in (12, 13):
        layer.kind = kind
        t = tensor((TQ, D))
        assert stub.ms_layer_forward(ctypes.byref(layer), ref(t), None, None, 0, ref(t), ctypes.byref(h), None) == L.MS_E_ARG


@pytest.mark.parametrize("kind", TRAINED)
def test_backward_refusals_leave_the_record_usable(stub, kind):
    c = Call(stub, kind)
    assert c.forward() == 0
    stub.attention_reset()
    assert c.backward(dy=None) == L.MS_E_NULL
    assert c.backward(mask=3) == L.MS_E_MASK             # no place for a gradient that was asked for
    H = c.a["y"].shape[1]
    assert c.backward(dy=out(T=TQ + 1, H=H)) == L.MS_E_SHAPE
    assert c.backward(dy=out(H=H, dtype="f32")) == L.MS_E_DTYPE
    stub.ms_testing_fail_next_workspace(1)
    assert c.backward() == L.MS_E_NOMEM
    assert stub.attention_log() == b""
    assert c.backward() == 0
    c.free()


@pytest.mark.parametrize("kind", KINDS)
def test_forward_without_memory(stub, kind):
    H = Call(stub, kind).a["x"].shape[1]
    c = Call(stub, kind, x=heads(H=H, strides=(2 * H * D, 2 * D, 2)))   # staged
    stub.ms_testing_fail_next_workspace(1)
    assert c.forward() == L.MS_E_NOMEM and not c.h.value
    assert stub.attention_log() == b"" and stub.stub_log() == b""
    assert c.forward() == 0
    c.free()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_other_layouts_are_staged(stub, kind, dtype):
    """A tensor of strided elements is copied in and out; one whose elements lie side by side
    only where its reader needs whole vectors (attention's rows, not the norms')."""
    shape = lambda c, n: tuple(c.a[n].shape[i] for i in range(3))
    c = Call(stub, kind, dtype)
    x, y = shape(c, "x"), shape(c, "y")
    apart = lambda s, addr: tensor(s, dtype, strides=(2 * s[1] * s[2], 2 * s[2], 2), addr=addr)
    c = Call(stub, kind, dtype, x=apart(x, FAKE), y=apart(y, OUT))
    assert c.forward() == 0
    assert stub.attention_log().count(b"pack;") == 1 and stub.stub_log() == b"copy4;"
    if kind in TRAINED:
        reset(stub)
        assert c.backward() == 0
        # dy; x (a norm's input, an attention's q), an attention's o; dx out
        assert stub.attention_log().count(b"pack;") == (3 if kind == "attention" else 2) and stub.stub_log() == b"copy4;"
        c.free()
    reset(stub)
    odd = tensor(x, dtype, strides=(x[1] * (D + 1), D + 1, 1))
    c = Call(stub, kind, dtype, x=odd)
    assert c.forward() == 0
    assert stub.attention_log().count(b"pack;") == (1 if kind in ("attention", "paged") else 0) and stub.stub_log() == b""
    c.free()


@pytest.mark.parametrize("strides,packs", [((HQ * D, D, 1), 0), ((D, TQ * D, 1), 0), ((0, D, 1), 1), ((HQ * D, 0, 1), 0), ((2 ** 23, D, 1), 0),
                                          ((2 ** 23 + 8, D, 1), 1), ((HQ * D + 4, D, 1), 1), ((D - 8, 2 ** 20, 1), 1)])
def test_rows_that_attention_reads_in_place(stub, strides, packs):
    c = Call(stub, "attention", x=heads(strides=strides), mask=0, kept=None)
    assert c.forward() == 0
    assert stub.attention_log().count(b"pack;") == packs


@pytest.mark.parametrize("addr,packs", [(FAKE + 16, 0), (FAKE + 8, 1)])
def test_unaligned_pointers_are_staged(stub, addr, packs):
    for kind in ("attention", "paged"):
        reset(stub)
        c = Call(stub, kind, x=heads(addr=addr), **(dict(mask=0, kept=None) if kind == "attention" else {}))
        assert c.forward() == 0
        assert stub.attention_log().count(b"pack;") == packs


@pytest.mark.parametrize("d", [1, 3, 31, 33, 255])
def test_odd_head_sizes_are_padded(stub, d):
    for dtype in ("bf16", "f32"):
        c = Call(stub, "attention", dtype, x=heads(D_=d, dtype=dtype), y=out(D_=d, dtype=dtype), **K(D_=d, dtype=dtype))
        assert c.forward() == 0 and stub.attention_log().count(b"pack;") == 3 and stub.stub_log() == b"copy4;"
        reset(stub)
        assert c.backward() == 0 and stub.attention_log().count(b"pack;") == 5 and stub.stub_log() == b"copy4;" * 3
        c.free()
        reset(stub)


@pytest.mark.parametrize("kind", KINDS)
def test_no_rows(stub, kind):
    c = Call(stub, kind)
    H = c.a["x"].shape[1]
    over = dict(x=heads(T=0, H=H, addr=None), y=heads(T=0, H=c.a["y"].shape[1], addr=None), n=0, pos=None, lengths=None, tables=None, kept=None)
    c = Call(stub, kind, **over)
    assert c.forward() == 0, stub.ms_last_error()
    if kind in TRAINED:
        assert c.backward() == 0
        c.free()


def test_queries_without_keys_and_keys_without_queries(stub):
    none = K(T=0, addr=None)
    c = Call(stub, "attention", **none)
    assert c.forward() == 0 and c.backward() == 0
    c.free()
    c = Call(stub, "attention", x=heads(T=0, addr=None), y=heads(T=0, addr=None), kept=None)
    assert c.forward() == 0 and c.backward() == 0
    c.free()


def test_caches_without_pages_or_heads_of_queries(stub):
    empty = dict(kp=pages(0, HK, PAGE, D, addr=None), vp=pages(0, HK, PAGE, D, addr=None), width=0, tables=None)
    assert Call(stub, "paged", **empty).forward() == 0
    assert Call(stub, "append", **empty).forward() == 0
    assert Call(stub, "append", qh=0, x=heads(H=2 * HK), y=None).forward() == 0
    assert Call(stub, "append", rows=FAKE, n=1).forward() == 0          # many tokens of one sequence


def test_tables_of_the_most_places(stub):
    assert Call(stub, "paged", width=2 ** 28 - 513).forward() == 0


@pytest.mark.parametrize("kind", TRAINED)
def test_backward_from_the_fixed_scratch(stub, kind):
    c = Call(stub, kind)
    assert c.forward() == 0
    stub.stub_reset()
    stub.ms_testing_fail_next_workspace(1)
    assert c.backward(entry="ms_layer_backward_noalloc") == 0
    assert stub.stub_log() == b"scratch;"
    stub.ms_testing_fail_next_workspace(0)
    c.free()


def test_in_place_without_a_record(stub):
    H = HQ + 2 * HK
    assert Call(stub, "append", y=heads(strides=(H * D, D, 1))).forward() == 0   # x's first heads
    assert Call(stub, "paged", y=heads()).forward() == 0
    for over in (dict(mask=0), dict(mask=1, norm=0, gq=None, gk=None)):   # what the backward reads is not overwritten
        c = Call(stub, "rotary", y=heads(H=HQ + HK), **over)
        assert c.forward() == 0
        if over["mask"]:
            assert c.backward() == 0
            c.free()
