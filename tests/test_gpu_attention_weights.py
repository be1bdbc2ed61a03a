"""Places that are seen with a weight of zero: an infinity there is 0 times an infinity, NaN, as the formulas
have it, wherever it lies in a tile.  (Only what is hidden takes no part.)"""
import math

import pytest
import torch

import paper_2404_12406_amd as ms
from test_gpu_attention import close, draw, reference, run

pytestmark = pytest.mark.gpu
CASES = pytest.mark.parametrize("dtype,D", [(t, D) for t in ("bf16", "f32") for D in (64, 128, 200)])
# keys in a tile with hidden places for some of the rows that see them, and in tiles without for others
N, AT = 300, 77


def inputs(D, dtype):
    """Scores that no query gives a weight to: -10^4 with key AT."""
    q, k, v, g = (draw((N, 2, D), dtype, i) for i in range(4))
    q[:, :, 0] = 1.0
    k[:, :, 0] = 0.0
    k[AT] = 0.0
    k[AT, :, 0] = -1e4 * D ** 0.5
    return q, k, v, g


@CASES
def test_a_value(D, dtype):
    q, k, v, g = inputs(D, dtype)
    refs, bars = reference(q, k, v, g, [N], [N], True, D ** -0.5, dtype)
    v[AT] = math.inf
    o = ms.layer_forward(ms.Attention(), q, k, v)[0]
    assert torch.isnan(o[AT + 1:]).all()          # (row AT sees keys before it, whose weights sum up to one)
    assert torch.isnan(o[AT]).all()
    close("o", o[:AT], refs[0][:AT], bars[0][:AT])
    # not causal: the hidden places are those past the last key
    for n in (AT + 1, AT + 5, 96, 128, N):
        o = ms.layer_forward(ms.Attention(causal=False), q[:40], k[:n], v[:n])[0]
        assert torch.isnan(o).all()


@CASES
def test_a_key(D, dtype):
    """Minus infinity with key AT: dS is 0 there, and dq the sum of 0 times it and the rest."""
    q, k, v, g = inputs(D, dtype)
    refs, bars = reference(q, k, v, g, [N], [N], True, D ** -0.5, dtype)
    k[AT, :, 0] = -math.inf
    for mask in (1, 7):
        dq = run(q, k, v, g, mask, ms.Attention())[1]
        assert torch.isnan(dq[AT:, :, 0]).all()
        close("dq", dq[:AT], refs[1][:AT], bars[1][:AT])
        close("other elements", dq[AT:, :, 1:], refs[1][AT:, :, 1:], bars[1][AT:, :, 1:])


@CASES
def test_a_gradient_and_a_query(D, dtype):
    """A row of g that is infinite, or of q: every key that the row sees has NaN, whatever its weight."""
    q, k, v, g = inputs(D, dtype)
    k[AT] = 0.0
    k[:, :, 0] = -1e4 * D ** 0.5
    k[0, :, 0] = 0.0                              # all but the first key are seen with a weight of zero
    at = 140
    refs, bars = reference(q, k, v, g, [N], [N], True, D ** -0.5, dtype)
    g2 = g.clone()
    g2[at] = math.inf
    for mask in (4, 7):
        dv = run(q, k, v, g2, mask, ms.Attention())[3]
        assert torch.isnan(dv[1:at + 1]).all() and torch.isinf(dv[0]).all()
        close("dv", dv[at + 1:], refs[3][at + 1:], bars[3][at + 1:])
