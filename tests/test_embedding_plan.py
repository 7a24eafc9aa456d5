"""The rules of the sorted embedding gradient (csrc/embedding_plan.h), compiled with the host compiler and checked without a GPU; and which kernels the
large batches of test_gpu_embedding_large.py run."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT = os.path.join(ROOT, "_build", "host_plan")
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")


@pytest.fixture(scope="module")
def plan():
    os.makedirs(OUT, exist_ok=True)
    so = os.path.join(OUT, "embedding.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so,
                           "-I", os.path.join(ROOT, "paper_2605_10501_amd", "csrc"), os.path.join(ROOT, "tests", "host_plan", "embedding_abi.cpp")])
    lib = C.CDLL(so)

    def call(n, vocab, vpr):
        out = (C.c_int * 6)()
        lib.embedding_plan(n, vocab, vpr, out)
        return dict(zip(("bits", "passes", "ipt", "blocks", "tile", "stream"), out))
    return call


def test_digits_cover_the_keys_and_workgroups_the_tokens(plan):
    for vocab in (1, 2, 511, 512, 513, 1024, 32000, 151936, 262143, 262144, 2**27 - 1, 2**31 - 2):
        for n in (1, 64, 4096, 4097, 131072, 131073, 524288, 524289, 1 << 24):
            p = plan(n, vocab, 16)
            assert p["bits"] <= 9 and (1 << (p["bits"] * p["passes"])) > vocab               # ids outside the table have the key `vocab`
            assert p["blocks"] * p["ipt"] * 1024 >= n if n > 4096 else p["blocks"] == 1
            assert p["blocks"] <= 1024


def test_the_large_batches_of_the_gpu_tests_take_the_large_kernels(plan):
    from test_gpu_embedding_large import CASES
    seen = set()
    for n, d, vocab, _, dtype, tile, stream in CASES:
        p = plan(n, vocab, d // (8 if dtype == "bf16" else 4))
        assert (p["tile"], bool(p["stream"])) == (tile, stream), (n, d, dtype)
        seen.add((dtype, tile, stream))
    # a bf16 and an fp32 kernel each: pieces of 32 places, dx read with and without the non-temporal policy
    assert {(t, 32, s) for t in ("bf16", "fp32") for s in (False, True)} <= seen


def test_small_pieces_are_never_read_past_the_caches(plan):
    """So that there is no kernel for both."""
    for n in (1, 4096, 20000, 32768, 1 << 20, 1 << 24):
        for vpr in (1, 16, 192, 1024, 4194304 // n, 4194304 // n + 1, 5000000 // n, 5000000 // n + 1):
            p = plan(n, 1000, max(vpr, 1))
            assert p["tile"] == 32 or not p["stream"]
