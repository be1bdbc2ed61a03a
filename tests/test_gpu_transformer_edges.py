"""The transformer layers at the edges of their ranges: no rows, rows by the
million, calls that keep nothing."""
import numpy as np
import pytest
import torch

import paper_2404_12406_amd as ms
from _gpu import TORCH_DT, guarded_empty, guards_intact

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", ["projections", "input"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_unit_of_no_rows(dtype, keep):
    """Its parameters' gradients are zeros, at widths that the contractions pad and from
    parameters that begin anywhere."""
    for D, F, off in ((513, 700, 0), (24, 41, 1), (2045, 2050, 1)):
        place = lambda *s: torch.ones(int(np.prod(s)) + off, dtype=TORCH_DT[dtype], device="cuda")[off:].view(s)
        x, W, b = torch.empty((0, D), dtype=TORCH_DT[dtype], device="cuda"), place(2 * F, D), place(2 * F)
        y, rec = ms.layer_forward(ms.GatedLinear("silu", keep), x, W, b, 7)
        outs = [guarded_empty(s, dtype) for s in ((0, D), (2 * F, D), (2 * F,))]
        ms.layer_backward(rec, torch.empty_like(y), *(o[0] for o in outs))
        torch.cuda.synchronize()
        for view, buf, guard in outs[1:]:
            assert not view.any() and guards_intact(buf, guard)


@pytest.mark.parametrize("dtype,rows", [("bf16", 2 ** 23 + 5), ("f32", 2 ** 22 + 3)])
def test_rows_by_the_million(dtype, rows):
    """More dz than 32-bit offsets reach in a tile's width of words (bf16: a dense prediction
    of some classes for every pixel): smaller pieces.  Bars: the gradients' of
    test_gpu_linear_cross_entropy.py; the fp32 sums of dW have some 1e6 terms a split, whose
    errors add up as their root, 2^-24 x 1e3 of the root of their squares' sum, which is dW's size."""
    D, V = 16, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, D, device="cuda", generator=g).to(TORCH_DT[dtype])
    W = torch.randn(V, D, device="cuda", generator=g).to(TORCH_DT[dtype])
    t = torch.randint(0, V, (rows,), device="cuda", generator=g)
    t[::5] = -100
    loss, rec = ms.layer_forward(ms.LinearCrossEntropy(t, reduction="sum"), x, W, None, 3)
    dx, dW, _ = ms.layer_backward(rec, torch.ones(1, device="cuda"))
    Wd, want, gW, worst, size = W.double(), 0.0, 0.0, 0.0, 0.0
    for i in range(0, rows, 2 ** 20):
        xi, ti = x[i:i + 2 ** 20].double(), t[i:i + 2 ** 20]
        live = ti != -100
        z = xi @ Wd.t()
        lse = torch.logsumexp(z, 1)
        pick = ti.clamp(min=0)[:, None]
        want += float(((lse - z.gather(1, pick)[:, 0]) * live).sum())
        z = torch.exp(z - lse[:, None])
        z.scatter_add_(1, pick, torch.full_like(z[:, :1], -1.0))
        z *= live[:, None]
        gx = z @ Wd
        gW = gW + z.t() @ xi
        worst, size = max(worst, float((dx[i:i + 2 ** 20].double() - gx).abs().max())), max(size, float(gx.abs().max()))
    bar = {"bf16": 2.0 ** -7, "f32": 5e-5}[dtype]
    assert abs(loss.item() - want) <= 2e-5 * abs(want)
    assert worst <= bar * size
    assert float((dW.double() - gW).abs().max()) <= (bar + 2.0 ** -14) * float(gW.abs().max())


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_modules_that_train_keep_nothing_where_no_gradient_can_follow(mode):
    from paper_2404_12406_amd import autograd as msa
    g = torch.Generator().manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    x, t = make(600, 64), torch.arange(600, device="cuda") % 50
    for m, args in ((msa.MSLayerNorm(make(64), make(64)), ()), (msa.MSGatedLinear(make(192, 64), make(192)), ()),
                    (msa.MSLinearCrossEntropy(make(50, 64), make(50)), (t,))):
        want = m(x, *args).detach()
        with mode():
            h = x + 0
            m(h, *args)
            torch.cuda.synchronize()
            before = torch.cuda.memory_allocated()
            torch.cuda.reset_peak_memory_stats()
            ms.ledger_reset()
            got = m(h, *args)
            assert torch.cuda.max_memory_allocated() - before <= got.untyped_storage().nbytes() + 512   # the output alone
            assert ms.ledger_read()[1] == ms.ledger_read()[0] == 0
        assert torch.equal(got, want)


def test_backward_on_another_stream_than_the_forward():
    """The records' buffers are not handed out again before that backward has read them."""
    g = torch.Generator().manual_seed(5)
    make = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    x, dy = make(4096, 256), make(4096, 512)
    one, t = torch.ones(1, device="cuda"), torch.arange(4096, device="cuda") % 3000
    for spec, W, gy, mask, kept in ((ms.GatedLinear(), make(1024, 256), dy, 1, "projections"),
                                    (ms.LinearCrossEntropy(t), make(3000, 256), one, 1, "grad"),
                                    (ms.LinearCrossEntropy(t), make(3000, 256), one, 2, "lse")):
        _, rec = ms.layer_forward(spec, x, W, None, mask)
        want = ms.layer_backward(rec, gy)
        other, here = torch.cuda.Stream(), torch.cuda.current_stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            _, rec = ms.layer_forward(spec, x, W, None, mask)
        n = rec.saved[kept].untyped_storage().nbytes()
        here.wait_stream(other)
        torch.cuda._sleep(20_000_000)   # the backward begins well after it is enqueued
        got = ms.layer_backward(rec, gy)
        with torch.cuda.stream(other):
            again = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert all(p is q or torch.equal(p, q) for p, q in zip(want, got)), kept
        del again


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cross_entropy_of_no_rows_whatever_the_workspace_holds(dtype, reduction):
    """Gradients are zeros: nothing that an earlier call left in the workspace reaches them."""
    make = lambda *s: torch.randn(*s).to(TORCH_DT[dtype]).cuda()
    spec = ms.LinearCrossEntropy(torch.empty(0, dtype=torch.int64, device="cuda"), reduction=reduction)
    for mask in (2, 3, 4, 6, 7):
        _, rec = ms.layer_forward(ms.GatedLinear(), make(64, 40), make(96, 40), None, 1)
        ms.layer_backward(rec, make(64, 48) * float("nan"))   # NaN from the workspace's beginning on
        _, rec = ms.layer_forward(spec, make(0, 40), make(421, 40), make(421), mask)
        grads = ms.layer_backward(rec, torch.ones(0 if reduction == "none" else 1, device="cuda"))
        assert not any(g.any() for g in grads if g is not None and g.numel())
