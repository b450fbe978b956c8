"""The attention of several queries and the sum behind a block on host threads under AddressSanitizer and UndefinedBehaviorSanitizer, as
test_cache_sanitized.py runs the operators on a paged cache."""
import os
import shutil
import subprocess
import sys

import pytest

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_several_queries_run_clean_under_sanitizers():
    from tests.cpu_emul import build_cache_cpu
    build_cache_cpu.build_sanitized()
    libs = [subprocess.run(["g++", f"-print-file-name={x}.so"], capture_output=True, text=True, check=True).stdout.strip() for x in ("libasan", "libubsan")]
    env = dict(os.environ, STTM_SANITIZED="1", LD_PRELOAD=":".join(libs), ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    some = ("f32-3-3-72 or bf16-17-1 or f16-4-2-80 or f32-5-5-24 or bf16-2-2-256 or bf16-7-1 or bf16-3-1-64 or outside or further or make_no_sense or f16-1-1-8 "
            "or empty or left_out or 520 or refusals")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_queries_cpu.py"), "-q", "-x", "-p", "no:cacheprovider",
                        "-k", some], capture_output=True, text=True, timeout=900, cwd=ROOT, env=env)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-6000:])
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
