"""The operators on a paged cache on host threads under AddressSanitizer and UndefinedBehaviorSanitizer, in a process of its own
that has libasan loaded first: reads and writes out of range, in the caller's buffers and in the kernels' own arrays."""
import os
import shutil
import subprocess
import sys

import pytest

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_paged_cache_runs_clean_under_sanitizers():
    from tests.cpu_emul import build_cache_cpu
    build_cache_cpu.build_sanitized()
    libs = [subprocess.run(["g++", f"-print-file-name={x}.so"], capture_output=True, text=True, check=True).stdout.strip() for x in ("libasan", "libubsan")]
    env = dict(os.environ, STTM_SANITIZED="1", LD_PRELOAD=":".join(libs), ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    some = "rope or 300-121 or 1100 or (5000 and ties) or 8200 or 6000 or without or outside or 136 or 160 or 257 or 17-1-64 or 33-1-40 or lengths1"
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_cache_small_cpu.py"), "-q", "-x", "-p", "no:cacheprovider", "-k", some],
                       capture_output=True, text=True, timeout=900, cwd=ROOT, env=env)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-6000:])
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
