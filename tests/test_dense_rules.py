"""The dense operators' rules on sizes, built for the host (tests/host/dense_rules.cpp)."""
import ctypes
import random
import subprocess

import pytest

from conftest import ROOT

FEW, SMALL, MID, LARGE = range(4)
# the tiles that a plan is laid out for, and the products that run over it (forward; backward)
PAIRS = [(FEW, FEW), (SMALL, SMALL), (MID, MID), (LARGE, LARGE), (LARGE, MID), (FEW, SMALL)]


@pytest.fixture(scope="module")
def dense_rules(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rules") / "libdenserules.so")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-Iinclude", "tests/host/dense_rules.cpp", "-o", out], cwd=ROOT, check=True)
    lib = ctypes.CDLL(out)
    lib.launched.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                             ctypes.POINTER(ctypes.c_int32)]
    lib.launched.restype = ctypes.c_int64
    return lib


def loads_of(rng):
    """Pairs an expert, uneven in several ways: one takes most, all just past a tile's height, any."""
    E = rng.choice([1, 2, 3, 8, 13, 16, 32, 64, 300])
    kind = rng.randrange(4)
    if kind == 0:
        loads = [1] * E
        loads[rng.randrange(E)] = rng.randint(1, 9 * E + 300)
    elif kind == 1:
        height = rng.choice([16, 32, 128, 256])
        loads = [rng.choice([0, 1, height + 1, 2 * height + 1]) for _ in range(E)]
    elif kind == 2:
        loads = [rng.randint(0, 40) for _ in range(E)]
    else:
        loads = [0] * E
        loads[rng.randrange(E)] = rng.randint(0, 3000)
    return loads


@pytest.mark.parametrize("plan,tile", PAIRS)
def test_the_grid_holds_every_tile_row_of_a_plan(dense_rules, plan, tile):
    rng = random.Random(plan * 10 + tile)
    split = ctypes.c_int32()
    height = dense_rules.height(plan)
    for _ in range(2000):
        loads = loads_of(rng)
        rows = dense_rules.launched(sum(loads), len(loads), plan, tile, ctypes.byref(split))
        planned = sum(-(-n // height) for n in loads)
        assert split.value * dense_rules.height(tile) >= height
        assert rows >= planned * split.value, (loads, rows, planned)
    # 16 experts, one with 97 of 127 pairs: 22 tile rows of 16
    assert dense_rules.launched(127, 16, FEW, SMALL, ctypes.byref(split)) >= 22


def test_launches_stay_within_the_threads_of_a_grid(dense_rules):
    x, y = ctypes.c_int64(), ctypes.c_int64()
    dense_rules.grid.argtypes = [ctypes.c_int64, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    dense_rules.grid.restype = ctypes.c_int64
    along = 1 << 21
    for blocks in (1, 8, 255, along - 1, along, along + 1, 1 << 22, (1 << 24) + 8, 1 << 28, 65535 * along):
        last = dense_rules.grid(blocks, ctypes.byref(x), ctypes.byref(y))
        assert x.value * 1024 < 1 << 32 and 1 <= y.value < 65536
        assert blocks <= last + 1 == x.value * y.value < blocks + along, blocks
        assert y.value == 1 or x.value == along
    dense_rules.grid(65535 * along + 1, ctypes.byref(x), ctypes.byref(y))
    assert x.value == 0  # refused
