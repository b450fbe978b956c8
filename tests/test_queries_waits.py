"""The assembly of the attention of several queries: a matrix product's result is not used before it is there, over every way through every
kernel (test_cache_waits.py says why this is looked at)."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_cache_waits import HIPCC, _least_distance

# Fewest wait states from a product of 32 x 32 to another use of its result, as the compiler keeps them everywhere else: eight passes (16-bit
# types, sixteen numbers a lane's row) and sixteen (fp32).
LEAST = {"x16_bf16": 12, "x16_f16": 12, "x2_f32": 18}

pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")


def test_results_of_matrix_products_are_waited_for(tmp_path):
    from paper_2507_07990_amd import build
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]

    def compiled(name):
        out = str(tmp_path / (name + ".s"))
        subprocess.run([HIPCC] + flags + ["--offload-device-only", "-S", os.path.join(build.CSRC, f"sttm_queries_{name}.hip"), "-o", out],
                       check=True, capture_output=True)
        return open(out).read()

    with ThreadPoolExecutor(3) as pool:
        texts = list(pool.map(compiled, ["f32", "bf16", "f16"]))
    least = {}
    for text in texts:
        kernels = 0
        for kernel in re.finditer(r"^(_ZN4sttm\S*k_query_tiles\S*):.*?^\.Lfunc_end\d+", text, re.S | re.M):
            kernels += 1
            lines = [x.split(";")[0].strip() for x in kernel[0].split("\n")]
            lines = [x for x in lines if x and (not x.startswith(".") or re.match(r"\.LBB\S+:", x))]
            labels = {x[:-1]: i for i, x in enumerate(lines) if x.endswith(":")}
            for i, line in enumerate(lines):
                if line.startswith("v_mfma"):
                    shape = re.match(r"v_mfma_f32_32x32(\S+)", line)[1]
                    least[shape] = min(least.get(shape, 99), _least_distance(lines, labels, i, most=24))
                    assert least[shape] >= LEAST[shape], (kernel[1], line, least)
        assert kernels == 40                                  # (five widths, two forms, two sources, rows full or not)
    assert set(least) == set(LEAST), least
