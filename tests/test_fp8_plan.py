"""The tile choice of the 8-bit products (csrc/fp8_plan.h), compiled with the host compiler and checked without a GPU."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT = os.path.join(ROOT, "_build", "host_plan")
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
FAST, PRECISE, SWIGLU = 0, 1, 2
TILES = {FAST: {256256, 256192, 128128, 128129, 64128, 64129, 64064}, PRECISE: {128128, 128129, 64128, 64129, 64064}, SWIGLU: {256256, 128128, 64128}}
ROWS = [65, 100, 200, 300, 420, 600, 777, 1100, 1500, 2049, 2900, 4096, 6000, 8192, 12000, 32768]
MATRICES = [(256, 256), (256, 688), (688, 256), (896, 4096), (1536, 1536), (2048, 5504), (2560, 8960), (4096, 2048), (4096, 11008), (6144, 4096), (8192, 2048),
            (11008, 2048), (22016, 4096)]


@pytest.fixture(scope="module")
def plan():
    os.makedirs(OUT, exist_ok=True)
    so = os.path.join(OUT, "fp8.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so,
                           "-I", os.path.join(ROOT, "paper_2605_10501_amd", "csrc"), os.path.join(ROOT, "tests", "host_plan", "fp8_abi.cpp")])
    lib = C.CDLL(so)
    lib.fp8_plan_us.restype = C.c_double
    lib.fp8_plan_us.argtypes = [C.c_int, C.c_int, C.c_long, C.c_long, C.c_long]
    lib.fp8_plan_tile.argtypes = [C.c_int, C.c_long, C.c_long, C.c_long]
    lib.fp8_plan_direct.argtypes = [C.c_long, C.c_long]
    return lib


@pytest.mark.parametrize("kind", [FAST, PRECISE, SWIGLU])
def test_the_choice_is_the_least_time_and_every_tile_is_one(plan, kind):
    seen = set()
    for m in ROWS:
        for n, k in MATRICES:
            kb = (k + 127) // 128
            us = {t: plan.fp8_plan_us(kind, t, m, n, kb) for t in TILES[kind]}
            tile = plan.fp8_plan_tile(kind, m, n, kb)
            assert tile in us and us[tile] == min(us.values()) and us[tile] > 0
            seen.add(tile)
    assert seen == TILES[kind]


def test_extreme_sizes_have_a_tile(plan):
    top = 2**31 - 1
    for kind in TILES:
        for m, n, kb in ((65, 16, 1), (top, 16, 1), (65, top, 1), (65, 16, 2**24), (top, top, 2**24)):
            assert plan.fp8_plan_tile(kind, m, n, kb) in TILES[kind]


def test_few_rows_go_without_tiles(plan):
    assert all(plan.fp8_plan_direct(m, n) for m in (1, 16) for n in (1, 16, 2**31 - 1))
    assert plan.fp8_plan_direct(64, 2048) and not plan.fp8_plan_direct(64, 2049) and not plan.fp8_plan_direct(65, 16)
