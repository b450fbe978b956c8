"""The attention of several queries, its kernels compiled for host threads (tests/cpu_emul), against the definitions in 64 bits:
indexing, masks, ragged sizes and refusals where there is no GPU."""
import ctypes
import os
import shutil

import pytest

from tests import cache_cases as C

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def bench():
    from paper_2507_07990_amd import binding
    from tests.cpu_emul import build_cache_cpu
    real = binding._lib
    binding._lib = binding._declare(ctypes.CDLL(build_cache_cpu.build_sanitized() if "STTM_SANITIZED" in os.environ else build_cache_cpu.build()))
    try:
        ctx = binding.Sttm(0, stream_ptr=0)
        ctx._device_index = -1                  # (host tensors)
        yield C.Bench(binding, ctx, "cpu")
        ctx.close()
    finally:
        binding._lib = real


from tests.query_tests import *  # noqa: E402,F401,F403  -- the tests themselves, on this file's `bench`
from tests.residual_tests import *  # noqa: E402,F401,F403
