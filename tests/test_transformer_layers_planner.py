"""What the transformer layers lay out, queried through the library's testing
hooks (no GPU: planning is host code)."""
import ctypes

import pytest

from paper_2404_12406_amd import _lib

F32, BF16 = _lib.MS_F32, _lib.MS_BF16


@pytest.fixture(scope="module")
def lib():
    return _lib.configure(ctypes.CDLL(_lib.LIB_PATH))


def gated(lib, dtype, rows, D, F, proj, aligned=1, mask=7):
    o = (ctypes.c_int64 * 4)()
    lib.ms_testing_gated_plan(dtype, rows, D, F, proj, aligned, mask, o)
    return dict(zip(("asked", "used", "D", "F"), o))


@pytest.mark.parametrize("proj", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gated_backward_stays_inside_its_workspace(lib, dtype, proj):
    """No rows among them: the gradients of W and b are still written, from the workspace
    that was asked for."""
    for rows in (0, 1, 7, 95, 96, 300, 5000):
        for D, F in ((24, 40), (513, 700), (516, 699), (2044, 2050), (4097, 4096)):
            for aligned in (0, 1):
                for mask in range(1, 8):
                    p = gated(lib, dtype, rows, D, F, proj, aligned, mask)
                    assert p["used"] <= p["asked"], (rows, D, F, aligned, mask, p)
