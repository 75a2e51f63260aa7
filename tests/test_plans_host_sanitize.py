"""The plans of the windowed attention's backward and of the shared prefixes, built for the CPU under AddressSanitizer and
UndefinedBehaviorSanitizer and driven by tests/sanitize/plans_driver.cpp, whose stand-ins for the launchers bound every
part of the scratch: tiles that several workgroups share by heads and by queries, chunks of sink tiles, packed and
unpacked column tiles of prefixes.  No GPU is used; the sanitizers apply to host code only."""
import os
import subprocess

import pytest

from test_cache_host_sanitize import CSRC, FLAGS, HIPCC, SAN


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_plans_under_asan_ubsan(tmp_path):
    objs = []
    for src in [os.path.join(CSRC, x) for x in ("ssba_cache_api.cpp", "ssba_window_api.cpp")] + \
            [os.path.join(SAN, "plans_driver.cpp")]:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, *FLAGS, "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    exe = tmp_path / "plans_driver"
    r = subprocess.run([HIPCC, "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        *objs, "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert r.stdout.strip() == "ok"
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
