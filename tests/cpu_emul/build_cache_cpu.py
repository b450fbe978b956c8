"""Builds tests/cpu_emul/libsttm_cache_cpu.so: the library with the operators on a paged cache, compiled with g++ against the
CPU stand-in for HIP in this folder (test infrastructure; the product is the hipcc build)."""
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

from tests.cpu_emul import build_cpu as base

LIB = os.path.join(base.HERE, "libsttm_cache_cpu.so")
# Short sequences take the ways of long ones: many chunks, all parts of an eviction, a wavefront with many rows of heads.
LIB_SMALL = os.path.join(base.HERE, "libsttm_cache_cpu_small.so")
SMALL = ["-DSTTM_CHUNK_MAX=32", "-DSTTM_ROPE_WAVES=1", "-DSTTM_ROPE_ONCE_BYTES=0", "-DSTTM_EVICT_LIST=128", "-DSTTM_EVICT_PART=256",
         "-DSTTM_EVICT_HERE=0"]
# ... under AddressSanitizer and UndefinedBehaviorSanitizer: any report ends the process that has it loaded (and libasan first).
LIB_SANITIZED = os.path.join(base.HERE, "libsttm_cache_cpu_sanitized.so")
SANITIZE = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
SOURCES = ["sttm_rope.hip", "sttm_attention.hip", "sttm_evict.hip"]


def _flags():
    return ["-fPIC", "-shared", "-fno-gnu-unique", "-include", os.path.join(base.HERE, "hip", "hip_cache.h")]


def build_sanitized() -> str:
    """(Its sources one by one, side by side: they take a minute or two.)"""
    if base._up_to_date(LIB_SANITIZED):
        return LIB_SANITIZED
    flags = ["g++", "-std=c++17", "-O1", "-g1", "-pthread", "-I", base.HERE, "-I", base.CSRC, "-Wno-unknown-pragmas", "-Wno-attributes"]
    sources = [os.path.join(base.CSRC, s) for s in base.SOURCES + SOURCES] + [os.path.join(base.HERE, "emul.cpp")]
    with tempfile.TemporaryDirectory() as folder, ThreadPoolExecutor(4) as pool:
        def compiled(source):
            out = os.path.join(folder, os.path.basename(source) + ".o")
            subprocess.run(flags + _flags() + SANITIZE + SMALL + ["-x", "c++", "-c", source, "-o", out], check=True)
            return out
        objects = list(pool.map(compiled, sources))
        subprocess.run(["g++", "-shared", "-pthread"] + SANITIZE + objects + ["-o", LIB_SANITIZED + ".part"], check=True)
    os.replace(LIB_SANITIZED + ".part", LIB_SANITIZED)
    return LIB_SANITIZED


def build(verbose: bool = False, small: bool = False) -> str:
    return base._compile(_flags() + (SMALL if small else []), [os.path.join(base.CSRC, s) for s in SOURCES], LIB_SMALL if small else LIB, verbose)


if __name__ == "__main__":
    print(build(verbose=True))
