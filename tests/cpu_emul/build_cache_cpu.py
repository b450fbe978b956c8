"""Builds tests/cpu_emul/libsttm_cache_cpu.so: the library with the operators on a paged cache, compiled with g++ against the
CPU stand-in for HIP in this folder (test infrastructure; the product is the hipcc build)."""
import os

from tests.cpu_emul import build_cpu as base

LIB = os.path.join(base.HERE, "libsttm_cache_cpu.so")
# Short sequences take the ways of long ones: many chunks, all parts of an eviction, a wavefront with many rows of heads.
LIB_SMALL = os.path.join(base.HERE, "libsttm_cache_cpu_small.so")
SMALL = ["-DSTTM_CHUNK_MAX=32", "-DSTTM_ROPE_WAVES=1", "-DSTTM_ROPE_ONCE_BYTES=0", "-DSTTM_EVICT_LIST=128", "-DSTTM_EVICT_PART=256",
         "-DSTTM_EVICT_HERE=0"]
SOURCES = ["sttm_rope.hip", "sttm_attention.hip", "sttm_evict.hip"]


def build(verbose: bool = False, small: bool = False) -> str:
    flags = ["-fPIC", "-shared", "-fno-gnu-unique", "-include", os.path.join(base.HERE, "hip", "hip_cache.h")]
    return base._compile(flags + (SMALL if small else []), [os.path.join(base.CSRC, s) for s in SOURCES], LIB_SMALL if small else LIB, verbose)


if __name__ == "__main__":
    print(build(verbose=True))
