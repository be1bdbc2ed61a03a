"""MSHeadNormRotary in a model that was converted to another type, forward and backward, against
the formulas in 64 bits; the bars are test_gpu_head_norm_rotary.py's."""
import pytest
import torch

import paper_2404_12406_amd as ms
from paper_2404_12406_amd import autograd as msa
from test_gpu_head_norm_rotary import compare, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how,dtype", [("bf16", "bf16"), ("there and back", "f32")])
def test_converted(how, dtype):
    """Positions to 100000: with frequencies of 8 bits an angle would be off by hundreds of radians."""
    x, gq, gk, gy, pos = inputs(50, 6, 64, "bf16", far=100000)
    freq = ms.rotary_frequencies(64, device="cuda")
    m = msa.MSHeadNormRotary(gq.float(), gk.float(), 4, freq.clone())
    m = m.bfloat16() if how == "bf16" else m.bfloat16().float()
    if dtype == "f32":
        x, gq, gk, gy = (t.float() for t in (x, gq, gk, gy))
    refs, bars = reference(x, gq, gk, gy, pos, freq, 4, True, False, dtype)
    x.requires_grad_()
    y = m(x, pos)
    y.backward(gy)
    compare([y.detach(), x.grad, m.weight_q.grad, m.weight_k.grad], refs, bars)
