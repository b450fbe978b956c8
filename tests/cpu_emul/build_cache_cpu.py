"""Builds tests/cpu_emul/libsttm_cache_cpu.so: the library with the operators on a paged cache, compiled with g++ against the
CPU stand-in for HIP in this folder (test infrastructure; the product is the hipcc build), under AddressSanitizer's and
UndefinedBehaviorSanitizer's checks if asked for."""
import os

from tests.cpu_emul import build_cpu as base

LIB = os.path.join(base.HERE, "libsttm_cache_cpu.so")
SOURCES = ["sttm_rope.hip", "sttm_attention.hip", "sttm_evict.hip"]


def build(verbose: bool = False) -> str:
    return base._compile(["-fPIC", "-shared", "-fno-gnu-unique", "-include", os.path.join(base.HERE, "hip", "hip_cache.h")],
                         [os.path.join(base.CSRC, s) for s in SOURCES], LIB, verbose)


if __name__ == "__main__":
    print(build(verbose=True))
