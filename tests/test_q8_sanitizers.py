"""The host code of the layer norm and the 8-bit products (argument checks, sizes, plans) under AddressSanitizer and
UndefinedBehaviorSanitizer: its refusals in a subprocess against the host-sanitized build.  No GPU is touched."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc not available")
def test_q8_abi_under_asan_and_ubsan():
    sys.path.insert(0, ROOT)
    from paper_2511_18672_amd import build as B

    lib = os.path.join(B.BUILD, "sanitize", "libsphinx.so")
    sources = glob.glob(os.path.join(B.CSRC, "*")) + glob.glob(os.path.join(B.INCLUDE, "*"))
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(s) for s in sources):
        lib = B.build_sanitized()
    env = dict(os.environ)
    env.update(SPHINX_LIBRARY=lib, LD_PRELOAD=B.sanitizer_runtime(), ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "not gpu", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_q8_oracle.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    print(out[-3000:])
    assert "runtime error" not in out and "AddressSanitizer" not in out
    assert r.returncode == 0
    assert " passed" in out
