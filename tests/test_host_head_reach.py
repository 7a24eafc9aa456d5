"""Plans of the losses at the end of a section at lm_heads and token counts whose gradients pass 4 GB (CPU only): csrc/head_host.cpp under the host sanitizers, driven by
tests/host_sanitizer/driver_head_reach.cpp."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import CLANG, CSRC, HERE, ROOT, SAN, _run

OUT = os.path.join(ROOT, "_build", "host_head_reach")


@pytest.mark.skipif(shutil.which("hipcc") is None or not os.path.exists(CLANG), reason="needs the ROCm compilers")
def test_what_a_product_reads_and_writes_lies_below_4_gb():
    os.makedirs(OUT, exist_ok=True)
    objs = []
    for src in [os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "head_host.cpp"), os.path.join(HERE, "driver_head_reach.cpp")]:
        obj = os.path.join(OUT, os.path.basename(src) + ".o")
        cmd = ["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-x", "hip", "-Wno-unused-value"]
        for f in SAN:
            cmd += ["-Xarch_host", f]
        _run(cmd + ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj])
        objs.append(obj)
    exe = os.path.join(OUT, "driver")
    _run([CLANG, *SAN, *objs, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and "head reach: OK" in r.stdout, r.stdout + r.stderr
