"""Which calls of attention's layers have tensors that share memory, and what becomes of them (no GPU:
stub launchers)."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

from paper_2404_12406_amd import _lib as L
from test_attention_host import D, FAKE, HK, HQ, OUT, TK, TQ, Call, ref, tensor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NATIVE = os.path.join(ROOT, "tests", "native")
NO, YES, UNKNOWN = 0, 1, 2
SIZE = {"bf16": 2, "f32": 4}


@pytest.fixture(scope="module")
def lib():
    os.makedirs(os.path.join(NATIVE, "_build"), exist_ok=True)
    so = os.path.join(NATIVE, "_build", "libmemsave_overlap.so")
    csrc = os.path.join(ROOT, "paper_2404_12406_amd", "csrc")
    tmp = so + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", os.path.join(ROOT, "include")]
                   + [os.path.join(csrc, f) for f in ("memsave.cpp", "blocks.cpp", "attention.cpp")]
                   + [os.path.join(NATIVE, f) for f in ("host_stub.cpp", "blocks_stub.cpp", "overlap.cpp")] + ["-o", tmp], check=True)
    os.replace(tmp, so)
    lib = L.configure(ctypes.CDLL(so))
    for f in ("attention_log", "attention_violations", "stub_log"):
        getattr(lib, f).restype = ctypes.c_char_p
    return lib


@pytest.fixture(autouse=True)
def clean(lib):
    lib.attention_reset()
    lib.stub_reset()
    yield
    assert lib.attention_violations() == b""


# ------------------------------------------------------------------ by elements
def places(t):
    e = {L.MS_BF16: 2, L.MS_F32: 4}[t.dtype]
    return {t.data + e * sum(i * t.stride[k] for k, i in enumerate(at)) for at in itertools.product(*(range(t.shape[k]) for k in range(3)))}


def test_shared_memory_by_elements(lib):
    """Against the elements' addresses: never wrong, and exact for slices of one buffer."""
    rng = random.Random(3)
    known = 0
    for _ in range(20000):
        T, H, d = rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 4)
        order = rng.choice([(H * d, d, 1), (d, T * d, 1), (2 * H * d, 2 * d, 2), (H * (d + 1), d + 1, 1), (0, d, 1)])
        def part():
            strides = order if rng.random() < 0.9 else (H * d + 1, d, 1)
            return tensor((rng.randint(0 if rng.random() < 0.1 else 1, T), rng.randint(1, H), rng.randint(1, d)), "f32", strides,
                          FAKE + 4 * rng.randint(0, 30))
        a, b = part(), part()
        got = lib.overlap_shared(ref(a), ref(b))
        assert got == lib.overlap_shared(ref(b), ref(a))
        if got != UNKNOWN:
            assert got == (YES if places(a) & places(b) else NO)
            known += 1
    assert known > 15000


HEADS = HQ + 2 * HK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices_of_one_projection(lib, dtype):
    part = lambda h, n, T=TQ: tensor((T, n, D), dtype, (HEADS * D, D, 1), FAKE + h * D * SIZE[dtype])  # noqa: E731
    q, k, v = part(0, HQ), part(HQ, HK), part(HQ + HK, HK)
    for a, b in itertools.combinations((q, k, v), 2):
        assert lib.overlap_shared(ref(a), ref(b)) == NO
    assert lib.overlap_shared(ref(q), ref(part(HQ - 1, 2))) == YES
    assert lib.overlap_shared(ref(q), ref(part(HEADS, HQ))) == YES     # the next rows' heads
    assert lib.overlap_shared(ref(q), ref(part(HEADS * TQ, HQ))) == NO
    assert lib.overlap_shared(ref(part(HQ, 1)), ref(part(HQ + 1, 1))) == NO
    assert lib.overlap_shared(ref(q), ref(tensor((TQ, HQ, D), dtype, (D, TQ * D, 1), FAKE + 4))) == YES
    assert lib.overlap_shared(ref(k), ref(tensor((1, 1, HQ * D), dtype, addr=FAKE))) == NO
    assert lib.overlap_shared(ref(q), ref(tensor((TQ, HQ, D), dtype, (HEADS * D, D, 1), FAKE + 1))) == UNKNOWN
    big = tensor((2 ** 20, 40, 40), dtype)
    assert lib.overlap_shared(ref(big), ref(tensor((1, 1, 1), dtype, addr=FAKE + (2 ** 20 * 1600 - 1) * SIZE[dtype]))) == YES


# ------------------------------------------------------------------ attention's backward
def backward(lib, mask, **places_):
    """Whether the gradients wait, for a call whose tensors lie where `places_` says."""
    at = dict(q=FAKE, k=FAKE + (1 << 30), v=FAKE + (2 << 30), o=OUT, g=OUT + (1 << 30), dq=OUT + (2 << 30), dk=OUT + (3 << 30), dv=OUT + (4 << 30))
    at.update(places_)
    q, k, v = (tensor((n, h, D), addr=at[x]) for x, n, h in (("q", TQ, HQ), ("k", TK, HK), ("v", TK, HK)))
    c = Call(lib, "attention", mask=mask, x=q, gq=k, gk=v, y=tensor((TQ, HQ, D), addr=at["o"]))
    assert c.forward() == 0
    g, dq, dk, dv = (tensor((n, h, D), addr=at[x]) for x, n, h in (("g", TQ, HQ), ("dq", TQ, HQ), ("dk", TK, HK), ("dv", TK, HK)))
    assert lib.ms_layer_backward(c.h, ref(g), *(ref(t) if mask >> i & 1 else None for i, t in enumerate((dq, dk, dv))), None) == 0
    c.free()
    return lib.overlap_noted()


@pytest.mark.parametrize("mask", range(1, 8))
def test_gradients_that_lie_where_the_backward_reads_wait(lib, mask):
    at = dict(q=FAKE, k=FAKE + (1 << 30), v=FAKE + (2 << 30), o=OUT, g=OUT + (1 << 30))
    assert backward(lib, mask) == 0
    for i, name in enumerate(("dq", "dk", "dv")):
        for on in at:
            read = on not in ("v", "o") or mask & 3   # dv alone reads neither
            want = bool(mask >> i & 1 and read)
            assert backward(lib, mask, **{name: at[on]}) == want, (name, on)
            assert backward(lib, mask, **{name: at[on] + 16 * D}) == want, (name, on)


def test_gradients_beside_what_the_backward_reads_do_not_wait(lib):
    """One buffer of rows that hold q, k, v and their gradients."""
    H = 2 * HEADS
    part = lambda T, h, n: tensor((T, n, D), "bf16", (H * D, D, 1), FAKE + h * D * 2)  # noqa: E731
    for shift, want in ((HEADS, 0), (HEADS - 1, 1), (0, 1)):
        c = Call(lib, "attention", x=part(TQ, 0, HQ), gq=part(TK, HQ, HK), gk=part(TK, HQ + HK, HK))
        assert c.forward() == 0
        g = tensor((TQ, HQ, D), addr=OUT + (1 << 30))
        assert lib.ms_layer_backward(c.h, ref(g), ref(part(TQ, shift, HQ)), ref(part(TK, shift + HQ, HK)), ref(part(TK, shift + HQ + HK, HK)),
                                     None) == 0
        assert lib.overlap_noted() == want
        c.free()


def test_stand_ins_are_apart(lib):
    """Rows that are staged, in and out, are read and written before and after the kernels."""
    odd = lambda T, H, a: tensor((T, H, D - 1), "bf16", addr=a)  # noqa: E731
    c = Call(lib, "attention", x=odd(TQ, HQ, FAKE), gq=odd(TK, HK, FAKE + 4096), gk=odd(TK, HK, FAKE + 8192), y=odd(TQ, HQ, OUT))
    assert c.forward() == 0
    assert lib.ms_layer_backward(c.h, ref(odd(TQ, HQ, OUT)), ref(odd(TQ, HQ, FAKE)), ref(odd(TK, HK, FAKE + 4096)), ref(odd(TK, HK, FAKE + 8192)),
                                 None) == 0
    assert lib.overlap_noted() == 0
    c.free()


# ------------------------------------------------------------------ head norms' backward
@pytest.mark.parametrize("norm", [1, 0])
def test_head_norm_gradients_that_cross_what_is_read_are_staged(lib, norm):
    H, n = HQ + HK, TQ * (HQ + HK) * D * 2
    over = {} if norm else dict(gq=None, gk=None, mask=1)

    def staged(dx, x=FAKE, dy=OUT, strides=None, **shape):
        c = Call(lib, "rotary", norm=norm, x=tensor((TQ, H, D), addr=x), y=tensor((TQ, H, D), addr=OUT + (1 << 30)), **over)
        assert c.forward() == 0
        lib.stub_reset()
        to = tensor((TQ, H, D), strides=strides, addr=dx)
        g = [tensor((D,), addr=OUT + (5 << 30) + (i << 20)) if norm else None for i in range(2)]
        assert lib.ms_layer_backward(c.h, ref(tensor((TQ, H, D), addr=dy)), ref(to), ref(g[0]), ref(g[1]), None) == 0
        c.free()
        return lib.stub_log() == b"copy4;"

    other = (D, TQ * D, 1)
    assert not staged(OUT + (2 << 30)) and not staged(OUT + (2 << 30), strides=other)
    assert not staged(OUT) and not staged(FAKE)                        # a head is written where it was read
    assert staged(OUT, strides=other) and staged(OUT + 2 * D) and staged(OUT + 2 * D * H) and staged(OUT - 2 * D)
    assert not staged(OUT + n) and not staged(OUT - n)
    for dx, strides in ((FAKE, other), (FAKE + 2 * D, None)):
        assert staged(dx, strides=strides) == bool(norm)               # a rotation alone does not read x


# ------------------------------------------------------------------ results of the forwards
def heads(T, H, addr, strides=None):
    return tensor((T, H, D), strides=strides, addr=addr)


ALL = (HEADS * D, D, 1)   # rows of queries, keys and values
ROW = HEADS * D * 2
CROSSING = [
    # an output that begins inside what other blocks read
    ("attention", dict(y=heads(TQ, HQ, FAKE + D * 2))), ("attention", dict(y=heads(TQ, HQ, FAKE + HQ * D * 2), mask=0)),
    ("attention", dict(y=heads(TQ, HQ, FAKE - HQ * D * 2))),
    ("attention", dict(x=heads(TQ, HQ, FAKE + (1 << 30)), y=heads(TQ, HQ, FAKE + D * 2))),   # k and v
    ("attention", dict(x=heads(TQ, HQ, FAKE, ALL), gq=heads(TQ, HK, FAKE + HQ * D * 2, ALL), gk=heads(TQ, HK, FAKE + (HQ + HK) * D * 2, ALL),
                       y=heads(TQ, HQ, FAKE + 2 * HK * D * 2, ALL))),
    ("rotary", dict(y=heads(TQ, HQ + HK, FAKE + D * 2), mask=0)), ("rotary", dict(y=heads(TQ, HQ + HK, FAKE + (HQ + HK) * D * 2))),
    ("rotary", dict(x=heads(TQ, HQ + HK, FAKE, ALL), y=heads(TQ, HQ + HK, FAKE + D * 2, ALL), mask=0)),
    ("append", dict(x=heads(TQ, HEADS, FAKE), y=heads(TQ, HQ, FAKE + D * 2, ALL))),
    ("append", dict(x=heads(TQ, HEADS, FAKE), y=heads(TQ, HQ, FAKE + ROW, ALL))), ("append", dict(y=heads(TQ, HQ, FAKE + 4 * D))),
    ("paged", dict(y=heads(TQ, HQ, FAKE + D * 2))), ("paged", dict(y=heads(TQ, HQ, FAKE - HQ * D * 2))),
]


@pytest.mark.parametrize("kind,over", CROSSING)
def test_results_that_cross_what_is_read_are_refused(lib, kind, over):
    c = Call(lib, kind, **over)
    assert c.forward() == L.MS_E_ARG, lib.ms_last_error()
    assert not c.h.value and lib.attention_log() == b"" and lib.stub_log() == b""


BESIDE = [
    # slices of one buffer: the results beside what is read
    ("attention", dict(x=heads(TQ, HQ, FAKE, (2 * HEADS * D, D, 1)), y=heads(TQ, HQ, FAKE + HEADS * D * 2, (2 * HEADS * D, D, 1)), mask=0,
                       gq=heads(TK, HK, OUT), gk=heads(TK, HK, OUT))),
    ("attention", dict(y=heads(TQ, HQ, FAKE + (1 << 20)), mask=0)),
    ("rotary", dict(x=heads(TQ, HQ + HK, FAKE, ALL), y=heads(TQ, HQ + HK, FAKE, ALL), mask=0)),
    ("append", dict(x=heads(TQ, HEADS, FAKE), y=heads(TQ, HQ, FAKE, ALL))),
    ("append", dict(x=heads(TQ, HEADS, FAKE, (2 * HEADS * D, D, 1)), y=heads(TQ, HQ, FAKE + HEADS * D * 2, (2 * HEADS * D, D, 1)))),
    ("paged", dict(y=heads(TQ, HQ, FAKE))), ("paged", dict(y=heads(TQ, HQ, FAKE + TQ * HQ * D * 2))),
]


@pytest.mark.parametrize("kind,over", BESIDE)
def test_results_beside_what_is_read_are_written(lib, kind, over):
    c = Call(lib, kind, **over)
    assert c.forward() == 0, lib.ms_last_error()


# ------------------------------------------------------------------ launches
@pytest.mark.parametrize("group,status", [(65535 * 32, 0), (65535 * 32 + 1, L.MS_E_UNSUPPORTED), (2 ** 23, L.MS_E_UNSUPPORTED)])
def test_query_heads_past_a_launchs_second_dimension_are_refused(lib, group, status):
    """Blocks of 32 query heads to a head of the cache are that dimension, up to 65535."""
    q, o = (tensor((1, group, 8), addr=a) for a in (FAKE, OUT))
    pages = tensor((9, 1, 8, 8))
    c = Call(lib, "paged", x=q, y=o, kp=pages, vp=pages, n=1)
    assert c.forward() == status
    assert lib.attention_log() == (b"" if status else b"paged;")
