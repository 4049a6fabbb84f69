"""The planners of the calls on a cache in 4 bits, built with AddressSanitizer and UndefinedBehaviorSanitizer and run on
random calls."""
import concurrent.futures
import os
import shutil
import subprocess

import pytest

from tests.test_sanitize import CSRC, HERE, HOST_SAN, ROOT, _run


def test_four_bit_planners_under_sanitizers(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if not hipcc:
        pytest.skip("hipcc not found")
    from paper_2504_14489_amd import build as hb
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops"] + HOST_SAN + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    # kv4_prefill.hip is part of the driver
    srcs = [os.path.join(CSRC, s) for s in hb.SOURCES if s != "kv4_prefill.hip"] + [os.path.join(HERE, "kv4_host.cpp")]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src).rsplit(".", 1)[0] + ".o"))
        res = subprocess.run([hipcc] + flags + ["-x", "hip", "-c", src, "-o", obj], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "kv4_host")
    res = subprocess.run([hipcc, "--offload-arch=gfx950"] + HOST_SAN + objs + ["-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    _run(exe, {"ASAN_OPTIONS": "detect_leaks=0"})
