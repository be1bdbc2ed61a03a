"""Cross entropy of targets that have nearly all of the probability, row by row against
the formulas in 64 bits: losses and gradients from 1 down to 1e-6 keep their leading digits.

Bars, relative to each row's own loss and gradient, from the arithmetic: both follow
from d, the log of the odds against the target, as exp(d) where they are small, so
their relative error is d's absolute one.  d is a difference of logits of some size Z, each
an fp32 sum of D products (2^-24 of Z for each rounding, sqrt(D) of them at random: 2^-21
Z at D = 264), of the log-sum that is kept (2^-25 Z) and of their sums: 2^-20 Z has a factor of
two of room.  Gradients have their own bars on top (test_gpu_linear_cross_entropy.py)."""
import pytest
import torch

import paper_2404_12406_amd as ms
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

OWN = {"f32": 5e-5, "bf16": 2.0 ** -7}


def inputs(M, V, dtype, shift, D=264, seed=1):
    """Targets whose logits stand 8 to 26 above the others' mean; every logit near `shift`."""
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(V, D, generator=g).to(TORCH_DT[dtype])
    t = torch.randperm(V, generator=g)[:M]
    Wt = W[t].double()
    x = Wt * (torch.linspace(8, 26, M)[:, None] / (Wt * Wt).sum(1, keepdim=True))
    b = torch.full((V,), float(shift)).to(TORCH_DT[dtype])
    return x.to(TORCH_DT[dtype]).cuda(), W.cuda(), b.cuda(), t.cuda(), (torch.rand(M, generator=g) + 0.5).cuda()


def reference(x, W, b, t, gl):
    x, W, b, gl = (v.double() for v in (x, W, b, gl))
    z = x @ W.t() + b
    pick = torch.arange(len(t), device="cuda")
    zt = z[pick, t]
    others = z.clone()
    others[pick, t] = -float("inf")
    d = torch.logsumexp(others, 1) - zt
    loss = torch.nn.functional.softplus(d, threshold=1e9)
    dz = torch.exp(others - (zt + loss)[:, None])
    dz[pick, t] = -torch.sigmoid(d)
    dz *= gl[:, None]
    return loss, dz @ W, dz.t() @ x, float(z.abs().max())


def worst(got, want):
    """The largest error of a row relative to its own largest value."""
    got, want = got.double(), want.reshape(len(want), -1)
    return float(((got.reshape(want.shape) - want).abs().amax(1) / want.abs().amax(1)).max())


@pytest.mark.parametrize("shift", [0, 80, -80])
@pytest.mark.parametrize("mask", [0, 1, 3])
@pytest.mark.parametrize("M,V", [(300, 30000), (16, 2000), (16, 60000), (2500, 3001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_losses_and_gradients(dtype, M, V, mask, shift):
    x, W, b, t, gl = inputs(M, V, dtype, shift)
    loss, dx, dW, size = reference(x, W, b, t, gl)
    assert float(loss.min()) < 2e-5 and float(loss.max()) > 0.1
    got, rec = ms.layer_forward(ms.LinearCrossEntropy(t, reduction="none"), x, W, b, mask)
    rel = size * 2.0 ** -20
    errs = {"loss": (worst(got, loss), rel)}
    if mask:
        if M == 300:
            assert ("grad" in rec.saved) == (mask == 1)   # both ways to the gradient are under test
        gx, gW, _ = ms.layer_backward(rec, gl)
        errs["dx"] = worst(gx, dx), OWN[dtype] + rel
        if mask & 2:   # the targets' rows of W (sums of some rows' terms, each as far off)
            errs["dW"] = worst(gW[t], dW[t]), 2 * (OWN[dtype] + rel)
    print(errs)
    assert all(e <= bar for e, bar in errs.values()), errs


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [1, 3])
def test_nothing_but_the_target(mask, dtype):
    """Every other word ruled out: no loss and no gradient, and no NaN."""
    x, W, b, t, gl = inputs(300, 30000, dtype, 0)
    t[:] = 77
    b[:] = -float("inf")
    b[77] = 1.0
    loss, rec = ms.layer_forward(ms.LinearCrossEntropy(t, reduction="none"), x, W, b, mask)
    gx, gW, _ = ms.layer_backward(rec, gl)
    assert not loss.any() and not gx.any() and (gW is None or not gW.any())
