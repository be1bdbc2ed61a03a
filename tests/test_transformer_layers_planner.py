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


# The contractions' operands: bytes below 2^32 less the last 16, which stand for "past
# the end", and less a load (bf16 by the general kernel's 32-bit indexes too).
MOST = {BF16: 2 ** 31 - 16, F32: 2 ** 30 - 8}
MOST_ROWS = 2 ** 27 - 8


def xent(lib, dtype, rows, D, V):
    o = (ctypes.c_int64 * 4)()
    lib.ms_testing_cross_entropy_plan(dtype, rows, D, V, o)
    return dict(zip(("words", "dz", "columns", "last"), o))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_piece_of_the_logits_has_32_bit_offsets(lib, dtype):
    for rows in (1, 8192, 2 ** 21, 2 ** 22, 2 ** 23 - 1, 2 ** 23, 10 ** 7, 16800000, 2 ** 25 + 1, 2 ** 26, MOST_ROWS):
        for V in (1, 7, 129, 150, 255, 256, 1000, 50000, 128001):
            p = xent(lib, dtype, rows, 8, V)
            assert 1 <= p["words"] <= V
            assert p["words"] == V or p["words"] % 8 == 0   # whole vectors of dz; pieces of b begin on 16 bytes
            assert p["dz"] <= MOST[dtype], (rows, V, p)
            if rows * V <= 2 ** 28:
                assert p["words"] == V


def test_padded_copies_have_32_bit_offsets(lib):
    """fp32 widths are padded to whole vectors only where the copies, and what is computed
    from them, stay below the contractions' limit (the general kernel's indexes end at 2^31)."""
    most = MOST[F32]
    for rows, D, V in ((2 ** 26, 3, 5), (2 ** 25 + 1, 31, 7), (2 ** 27 - 8, 1, 3), (100, 737, 2880000), (96, 5, 2 ** 27), (777, 514, 10007),
                       (2 ** 25 - 1, 5, 9)):
        p = xent(lib, F32, rows, D, V)
        assert p["columns"] == D or max(rows, p["words"]) * p["columns"] <= most, (rows, D, V, p)
        assert p["last"] == V - (V - 1) // p["words"] * p["words"] or max(p["last"] * p["columns"], rows * p["last"],
                                                                       rows * p["columns"]) <= most
    for rows, D, F in ((2 ** 27, 1, 1), (2 ** 26 + 1, 3, 5), (2 ** 25, 30, 15), (100, 9001, 60001), (1001, 515, 1366), (96, 2 ** 21 + 1, 500)):
        p = gated(lib, F32, rows, D, F, 0)
        assert (p["D"], p["F"]) == (D, F) or max(rows * p["D"], rows * 2 * p["F"], 2 * p["F"] * p["D"]) <= most, (rows, D, F, p)
    assert xent(lib, F32, 777, 514, 10007)["columns"] == 544 and gated(lib, F32, 1001, 515, 1366, 0)["D"] == 544


def test_widened_logits_fit_the_contractions_that_know_of_them(lib):
    """Rows of W past the last word are known to the fp32 contraction alone, not to the
    general one that takes larger operands (the first: x has 2^30 - 4 elements)."""
    widened = 0
    for rows, D, V in ((6242685, 172, 31), (6242600, 172, 31), (33554431, 32, 31), (33554430, 4, 29), (2 ** 20, 900, 1027)):
        p = xent(lib, F32, rows, D, V)
        if p["last"] != V - (V - 1) // p["words"] * p["words"]:
            widened += 1
            assert max(rows * p["columns"], p["last"] * p["columns"], rows * p["last"]) <= MOST[F32], (rows, D, V, p)
    assert widened > 1
