"""The cases of test_paged_edges.py against the host code under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only), with the library that
test_host_sanitizers.py builds."""
import os
import subprocess
import sys

import pytest

import test_host_sanitizers as H


@pytest.mark.skipif(os.environ.get("STRUCTKV_TEST_LIB") is not None, reason="already inside the sanitizer run")
def test_paged_edges_under_asan_ubsan():
    asan = subprocess.run(["gcc", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(asan) or not os.path.exists(asan):
        pytest.skip("no libasan.so in this toolchain")
    H._build_host_library()
    env = dict(os.environ, STRUCTKV_TEST_LIB=H.HOST_LIB, OMP_NUM_THREADS="4", LD_PRELOAD=":".join(x for x in (os.environ.get("LD_PRELOAD"), asan) if x),
               ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:abort_on_error=0:exitcode=97",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1:exitcode=98")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
                        os.path.join(H.ROOT, "tests", "test_paged_edges.py")], cwd=H.ROOT, env=env, capture_output=True, text=True, timeout=1500)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert r.returncode == 0 and " passed" in out and "skipped" not in out, out[-4000:]
