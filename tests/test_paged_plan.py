"""How paged attention divides a sequence's keys over blocks, over the range of tables that its
entry point takes (host arithmetic, no GPU)."""
import ctypes
import os
import random
import subprocess

import pytest

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")
MOST = 2 ** 31 - 1 - 4096   # places of a table


@pytest.fixture(scope="module")
def plan():
    os.makedirs(os.path.join(NATIVE, "_build"), exist_ok=True)
    so = os.path.join(NATIVE, "_build", "libpaged_plan.so")
    tmp = so + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wall", os.path.join(NATIVE, "paged_plan.cpp"), "-o", tmp], check=True)
    os.replace(tmp, so)
    lib = ctypes.CDLL(so)

    def of(n, group, Hk, page, width):
        out = (ctypes.c_int64 * 2)()
        lib.paged_plan(n, group * Hk, Hk, page, width, out)
        return out[0], out[1]

    return of


def check(plan, n, group, Hk, page, width):
    room = page * width
    splits, per = plan(n, group, Hk, page, width)
    assert splits >= 1 and per >= 128 and per % 128 == 0
    assert splits * per >= room, "keys of no block"
    assert (splits - 1) * per < max(room, 1), "blocks without keys in a full table"
    assert per < 2 ** 31 and splits < 2 ** 31


SIZES = [1, 2, 31, 64, 100, 255, 4096]


@pytest.mark.parametrize("page,width", [(1, 0), (1, 1), (16, 1), (5, 77), (16, 8192), (64, 2048), (1, 2 ** 30), (2 ** 20, 1023), (2 ** 20, 1024),
                                        (2 ** 20, 1025), (2 ** 20, 2047), (1, MOST), (MOST, 1), (65536, 32767)])
def test_every_place_has_a_block(page, width, plan):
    assert page * width <= MOST
    for n in SIZES:
        for Hk in (1, 2, 8, 40):
            for group in (1, 32, 33, 100):
                check(plan, n, group, Hk, page, width)


def test_every_place_has_a_block_anywhere(plan):
    rng = random.Random(5)
    for _ in range(20000):
        page = int(2 ** rng.uniform(0, 30.99))
        width = int(2 ** rng.uniform(0, 30.99)) % (MOST // page + 1)
        check(plan, int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(0, 6)), page, width)
