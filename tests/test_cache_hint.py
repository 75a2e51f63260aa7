"""The cache's host layer (ssba_cache_api.cpp) built for the CPU and driven by tests/sanitize/cache_hint_driver.cpp:
the length hint of a batch decides how work is split, never whether a call is accepted.  No GPU is used."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_15684_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_the_hint_decides_nothing_but_the_split(tmp_path):
    exe, objs = tmp_path / "hint", []
    for src in (os.path.join(CSRC, "ssba_cache_api.cpp"), os.path.join(ROOT, "tests", "sanitize", "cache_hint_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                            "-I", CSRC, "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([HIPCC, *objs, "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout + r.stderr)[-4000:]
