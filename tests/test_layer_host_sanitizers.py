"""The host checks of the position-wise entry points against the build whose host
code is instrumented (see test_host_sanitizers.py), in a child process (CPU only)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN_LIB = os.path.join(ROOT, "paper_2608_00938_amd", "_build", "libgrace_hostsan.so")

RUN = """
import sys
sys.path.insert(0, {root!r})
from paper_2608_00938_amd import grace as G
G._LIB_PATH = {lib!r}
import pytest
sys.exit(pytest.main([{tests!r}, "-q", "-p", "no:cacheprovider", "-m", "not gpu"]))
"""


@pytest.mark.skipif(not os.path.exists(SAN_LIB), reason="host-sanitizer build not present")
def test_layer_host_checks_under_sanitizers():
    from paper_2608_00938_amd import build_hostsan
    env = dict(os.environ, LD_PRELOAD=build_hostsan.asan_runtime(), HIP_VISIBLE_DEVICES="",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    tests = os.path.join(ROOT, "tests", "test_layer_host.py")
    p = subprocess.run([sys.executable, "-c", RUN.format(root=ROOT, lib=SAN_LIB, tests=tests)], env=env,
                       capture_output=True, text=True, timeout=600, cwd=ROOT)
    out = p.stdout + p.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
    assert p.returncode == 0, out[-4000:]
    assert " passed" in p.stdout, out[-2000:]
