"""The attention kernels' own assembly: a matrix product's result is not used before it is there.

Such a result may be read a number of cycles after the product was issued, and the compiler puts the waits in between. Where a
branch stood between the two it put none (ROCm 7.2, gfx950), and fp32 results came out wrong: the sources keep branches
out of there, and this looks whether it worked, over every way through every kernel."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Fewest wait states from a product of eight passes (fp32) or four passes of this shape to another use of its result, as the
# compiler itself keeps them everywhere else.
LEAST = {"f32": 10, "16": 8}

pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")


def _registers(word):
    m = re.match(r"([va])\[(\d+):(\d+)\]$", word)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.match(r"([va])(\d+)$", word)
    return {(m[1], int(m[2]))} if m else set()


def _least_distance(lines, labels, at, most=20):
    """Wait states from the product in lines[at] to the first use of its result, other than as what a product adds to."""
    result = _registers(re.split(r"[ ,]+", lines[at])[1])
    least, todo, seen = most, [(at + 1, 0)], set()
    while todo:
        i, waited = todo.pop()
        while i < len(lines) and waited < least and (i, waited) not in seen:
            seen.add((i, waited))
            words = re.split(r"[ ,]+", lines[i])
            i += 1
            if words[0].endswith(":"):
                continue
            if words[0] == "s_endpgm":
                break
            if words[0] == "s_nop":
                waited += int(words[1], 0) + 1
                continue
            if words[0].startswith("s_cbranch") or words[0] == "s_branch":
                if words[1] in labels:
                    todo.append((labels[words[1]], waited + 1))
                if words[0] == "s_branch":
                    break
            elif words[0].startswith(("v_", "ds_", "global_", "buffer_")):
                product = words[0].startswith("v_mfma")
                used = set().union(*[_registers(w) for w in (words[2:4] if product else words[1:])])
                if used & result:
                    least = min(least, waited)
                    break
                if product and _registers(words[1]) & result:
                    break
            waited += 1
    return least


def test_results_of_matrix_products_are_waited_for(tmp_path):
    from paper_2507_07990_amd import build
    out = str(tmp_path / "attention.s")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC] + flags + ["--offload-device-only", "-S", os.path.join(build.CSRC, "sttm_attention.hip"), "-o", out],
                   check=True, capture_output=True)
    text, products = open(out).read(), 0
    for kernel in re.finditer(r"^(_ZN4sttm\S*k_paged_attention\S*):.*?^\.Lfunc_end\d+", text, re.S | re.M):
        lines = [x.split(";")[0].strip() for x in kernel[0].split("\n")]
        lines = [x for x in lines if x and (not x.startswith(".") or re.match(r"\.LBB\S+:", x))]
        labels = {x[:-1]: i for i, x in enumerate(lines) if x.endswith(":")}
        for i, line in enumerate(lines):
            if line.startswith("v_mfma"):
                products += 1
                least = LEAST["f32" if "x4_f32" in line else "16"]
                assert _least_distance(lines, labels, i) >= least, (kernel[1], line)
    assert products > 1000
