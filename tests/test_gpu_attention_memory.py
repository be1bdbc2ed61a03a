"""Gradients of attention and of head norms written where their backward reads: on q, k, v, o or
the gradient of the output, in the same layout or another.  Every result has the bits that it has
in memory of its own (each is the same sum, rounded once)."""
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import api
from test_gpu_attention import draw, starts

pytestmark = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])

# (rows of the sequences, query heads, heads of keys, elements of a head): keys divided over blocks;
# blocks enough; eight waves a block, dk and dv in kernels of their own; heads in two kernels; staged rows
SHAPES = [([700], 4, 2, 64), ([300, 40, 900, 1], 8, 8, 64), ([2500, 2500], 8, 4, 128), ([500, 90], 4, 4, 200), ([130, 77], 2, 2, 33)]


def inputs(lens, Hq, Hk, D, dtype):
    T = sum(lens)
    return [draw((T, h, D), dtype, i) for i, h in enumerate((Hq, Hk, Hk, Hq))]


def apart(spec, q, k, v, g, mask):
    o, rec = ms.layer_forward(spec, q, k, v, mask)
    return o, ms.layer_backward(rec, g)


def same(got, want):
    for a, b in zip(got, want):
        assert (a is None) == (b is None)
        if b is not None:
            assert torch.isfinite(b).all() and torch.equal(a, b)


@DTYPES
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("mask", range(1, 8))
def test_gradients_on_the_inputs(mask, shape, dtype):
    q, k, v, g = inputs(*shape, dtype)
    spec = ms.Attention(starts(shape[0]))
    _, want = apart(spec, q, k, v, g, mask)
    q, k, v = (t.clone() for t in (q, k, v))
    _, rec = ms.layer_forward(spec, q, k, v, mask)
    same(ms.layer_backward(rec, g, *(t if mask >> i & 1 else None for i, t in enumerate((q, k, v)))), want)


@DTYPES
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients_on_one_projection(shape, causal, dtype):
    """q, k and v as one Linear wrote them, their gradients as its backward will read them."""
    q, k, v, g = inputs(*shape, dtype)
    Hq, Hk = shape[1:3]
    spec = ms.Attention(starts(shape[0]), causal=causal)
    _, want = apart(spec, q, k, v, g, 7)
    p = torch.cat([q, k, v], 1)
    parts = lambda: (p[:, :Hq], p[:, Hq:Hq + Hk], p[:, Hq + Hk:])  # noqa: E731
    _, rec = ms.layer_forward(spec, *parts(), 7)
    same(ms.layer_backward(rec, g, *parts()), want)


@DTYPES
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] == s[2]])
@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("on", ["g", "o"])
def test_a_gradient_on_the_outputs_gradient_or_the_output(on, which, shape, dtype):
    q, k, v, g = inputs(*shape, dtype)
    spec = ms.Attention(starts(shape[0]))
    _, want = apart(spec, q, k, v, g, 7)
    o, rec = ms.layer_forward(spec, q, k, v, 7)
    to = [None] * 3
    to[which] = g if on == "g" else o
    same(ms.layer_backward(rec, g, *to), want)


@DTYPES
@pytest.mark.parametrize("rows", [1, 40, 128])
def test_gradients_some_rows_further(rows, dtype):
    """Each gradient begins `rows` rows after what it lies on."""
    q, k, v, g = inputs([700], 4, 4, 64, dtype)
    spec = ms.Attention()
    _, want = apart(spec, q, k, v, g, 7)
    room = [torch.cat([t, torch.zeros_like(t[:rows])]) for t in (q, k, v)]
    _, rec = ms.layer_forward(spec, *(t[:700] for t in room), 7)
    same(ms.layer_backward(rec, g, *(t[rows:] for t in room)), want)


@DTYPES
def test_a_prepared_call_in_place(dtype):
    """Forward and backward several times over other inputs, the gradients on the inputs."""
    shape = ([300, 40, 90], 4, 2, 64)
    bufs = [torch.empty_like(t) for t in inputs(*shape, dtype)]
    q, k, v, g = bufs
    spec = ms.Attention(starts(shape[0]))
    call = api.PreparedLayer(spec, q, k, v, 7, grad_y=g, grad_x=q, grad_W=k, grad_b=v)
    for seed in range(3):
        for i, t in enumerate(bufs):
            t.copy_(draw(t.shape, dtype, 10 * seed + i))
        o, want = apart(spec, q, k, v, g, 7)
        call.forward()
        call.backward()
        same([call.y, q, k, v], [o, *want])


def test_a_prepared_call_of_its_own():
    """The same with gradients in memory of their own, and eager calls between."""
    q, k, v, g = inputs([300, 40, 90], 4, 2, 64, "bf16")
    spec = ms.Attention(starts([300, 40, 90]))
    grads = [torch.empty_like(t) for t in (q, k, v)]
    call = api.PreparedLayer(spec, q, k, v, 7, grad_y=g, grad_x=grads[0], grad_W=grads[1], grad_b=grads[2])
    for seed in range(3):
        for i, t in enumerate((q, k, v, g)):
            t.copy_(draw(t.shape, "bf16", 10 * seed + i))
        call.forward()
        o, want = apart(spec, q, k, v, g, 7)
        call.backward()
        same([call.y, *grads], [o, *want])

@DTYPES
def test_in_place_without_allocation(dtype):
    import ctypes
    from paper_2404_12406_amd import _lib
    q, k, v, g = inputs([300, 40, 90], 4, 2, 64, dtype)
    spec = ms.Attention(starts([300, 40, 90]))
    _, want = apart(spec, q, k, v, g, 7)
    _, rec = ms.layer_forward(spec, q, k, v, 7)
    assert _lib.load().ms_layer_backward_noalloc(rec._h, *(ctypes.byref(api.tensor_desc(t)) for t in (g, q, k, v)), api._stream(q.device)) == 0
    same((q, k, v), want)


@DTYPES
def test_graph_replays_in_place(dtype):
    """dq where o was, dk and dv where k and v are copied to: replays with other inputs, eager calls between."""
    shape = ([300, 40, 90], 4, 2, 64)
    q, k, v, g = inputs(*shape, dtype)
    spec = ms.Attention(starts(shape[0]))

    def step():
        k2, v2 = k.clone(), v.clone()
        o, rec = ms.layer_forward(spec, q, k2, v2, 7)
        return ms.layer_backward(rec, g, o, k2, v2)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step()
    torch.cuda.synchronize()
    for i in range(3):
        for j, t in enumerate((q, k, v, g)):
            t.copy_(draw(t.shape, dtype, 20 + 10 * i + j))
        graph.replay()
        torch.cuda.synchronize()
        same(outs, apart(spec, q, k, v, g, 7)[1])


# ------------------------------------------------------------------ head norms
@DTYPES
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("where", ["dy", "dy turned over", "dy a row on", "dy a head on", "x", "x turned over"])
@pytest.mark.parametrize("D,R", [(64, 64), (90, 36), (33, 30)])
def test_head_norm_gradients_on_what_is_read(D, R, where, norm, dtype):
    T, H = 60, 6
    x, dy = draw((T, H, D), dtype, 0, 1.5), draw((T, H, D), dtype, 1)
    gq, gk = (1 + draw((D,), dtype, 2 + i, 0.3) if norm else None for i in range(2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 37
    spec = ms.HeadNormRotary(pos, ms.rotary_frequencies(R, device="cuda"), 4, norm)
    mask = 7 if norm else 1
    want = ms.layer_backward(ms.layer_forward(spec, x, gq, gk, mask)[1], dy)
    room = torch.zeros((T + 1) * H * D, dtype=x.dtype, device="cuda")
    room[:T * H * D] = (dy if where[0] == "d" else x).flatten()
    at = room[:T * H * D].view(T, H, D)
    if where[0] == "d":
        dy = at
    else:
        x = at
    to = {"turned over": room[:T * H * D].view(H, T, D).transpose(0, 1), "a row on": room[H * D:].view(T, H, D),
          "a head on": room[D:][:T * H * D].view(T, H, D)}.get(where.partition(" ")[2], at)
    _, rec = ms.layer_forward(spec, x, gq, gk, mask)
    same(ms.layer_backward(rec, dy, to), want)
