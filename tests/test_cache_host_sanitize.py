"""The cache's host layer (ssba_cache_api.cpp) built for the CPU under
AddressSanitizer and UndefinedBehaviorSanitizer and driven by
tests/sanitize/cache_driver.cpp, whose stand-ins for the launchers check grid
sizes, workspace bounds and plans for 60 000 descriptors at the edges of the
integer ranges.  No GPU is used; the sanitizers apply to host code only."""
import os
import subprocess

import pytest

from test_host_sanitize import CSRC, FLAGS, HIPCC, SAN


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_cache_host_layer_under_asan_ubsan(tmp_path):
    objs = []
    for src in (os.path.join(CSRC, "ssba_cache_api.cpp"), os.path.join(SAN, "cache_driver.cpp")):
        obj = tmp_path / (os.path.basename(src) + ".o")
        r = subprocess.run([HIPCC, *FLAGS, "-c", src, "-o", str(obj)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
        objs.append(str(obj))
    exe = tmp_path / "cache_driver"
    r = subprocess.run([HIPCC, "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        *objs, "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert r.stdout.strip() == "ok"
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
