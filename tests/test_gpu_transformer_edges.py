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
