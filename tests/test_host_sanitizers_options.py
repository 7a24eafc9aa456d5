"""Sections with options under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only): their workspace plan and the order of their calls, as
test_host_sanitizers.py does it for sections without."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import CLANG, CSRC, HERE, ROOT, SAN, _run

OUT = os.path.join(ROOT, "_build", "host_sanitizer_options")


@pytest.mark.skipif(shutil.which("hipcc") is None or not os.path.exists(CLANG), reason="needs the ROCm compilers")
def test_sections_with_options_under_address_and_ub_sanitizers():
    os.makedirs(OUT, exist_ok=True)
    objs = []
    for src in [*(os.path.join(CSRC, f) for f in ("api.cpp", "kd_host.cpp", "column_work.cpp", "section.hip", "section_options.hip")),
                *(os.path.join(HERE, f) for f in ("driver_options.cpp", "fake_backend.cpp", "fake_options.cpp"))]:
        obj = os.path.join(OUT, os.path.basename(src) + ".o")
        cmd = ["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-x", "hip", "-Wno-unused-value"]
        for f in SAN:                                        # host pass only: each -fsanitize= directly after -Xarch_host
            cmd += ["-Xarch_host", f]
        _run(cmd + ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj])
        objs.append(obj)
    exe = os.path.join(OUT, "driver")
    _run([CLANG, *SAN, *objs, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and "host sanitizer driver: OK" in r.stdout, r.stdout + r.stderr
