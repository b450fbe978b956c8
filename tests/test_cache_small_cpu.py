"""The operators on a paged cache on host threads, built so that small inputs take the ways of large ones: sequences of many
chunks (more than a wavefront joins in one go), evictions by many workgroups with a list that holds few slots, wavefronts that
have many rows of heads and write past the caches."""
import ctypes
import os
import shutil

import pytest
import torch

from tests import cache_cases as C

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def bench():
    from paper_2507_07990_amd import binding
    from tests.cpu_emul import build_cache_cpu
    real = binding._lib
    binding._lib = binding._declare(ctypes.CDLL(build_cache_cpu.build_sanitized() if "STTM_SANITIZED" in os.environ else build_cache_cpu.build(small=True)))
    try:
        ctx = binding.Sttm(0, stream_ptr=0)
        ctx._device_index = -1                  # (host tensors)
        yield C.Bench(binding, ctx, "cpu")
        ctx.close()
    finally:
        binding._lib = real


# -- the tests themselves, on this file's `bench`
from tests.cache_tests import (test_cache_evict, test_cache_evict_leaves_whole_tables_where_numbers_occur_twice,  # noqa: E402,F401
                               test_cache_evict_without_slots, test_paged_attention, test_paged_attention_with_pages_outside_of_the_pool,
                               test_qk_norm_rope, test_qk_norm_rope_without_a_cache)


@pytest.mark.parametrize("dtype,H,K,lengths,bias_kind", [("bf16", 3, 1, (2500, 9), ""), ("f32", 1, 1, (2100,), "counts"), ("f16", 17, 1, (2200,), "counts"),
                                                         ("bf16", 2, 2, (9000,), ""), ("f32", 3, 1, (2300, 0), "")])
def test_paged_attention_of_very_many_chunks(bench, dtype, H, K, lengths, bias_kind):
    """More than 256 chunks to join; chunks of 8 slots and, from 4,096 slots in all rows on, of 16."""
    gen, d, page = torch.Generator().manual_seed(sum(lengths)), 8, 64
    kv, table = C.pool(gen, dtype, K, d, page, lengths)
    B, cap = len(lengths), max(lengths)
    bias = None
    if bias_kind:
        bias = torch.exp(torch.randn(B, K, cap, generator=gen)).ceil().log()
        bias[torch.rand(B, K, cap, generator=gen) < 0.3] = -C.INF
    q = (torch.randn(B, H, d, generator=gen) * 2).to(C.TYPES[dtype])
    q[:, 0] *= 8                                           # (the largest score is rare, and chunks' maxima far apart)
    win, lens = torch.rand(B, K, cap, generator=gen), torch.tensor(lengths, dtype=torch.int32)
    want = C.attention_reference(q, *kv, table, lens, page, d ** -0.5, bias, win, torch.zeros(B, K, cap), dtype)
    got = C.run_attention(bench, q, kv, "pages", table, lens, d ** -0.5, bias, win, torch.zeros(B, K, cap))
    for name, g, w in zip(("out", "lse", "weights"), got, want):
        C.close(g, *w, what=name)
