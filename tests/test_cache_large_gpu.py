"""The operators on a paged cache on the GPU at sizes on both sides of every rule that goes by size, against the definitions in
64 bits."""
import pytest
import torch

from tests import cache_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bench(lib):
    return C.Bench(lib, lib.Sttm(0), "cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("dtype,n,H,K,d,sections,interleaved", [
    ("bf16", 2100, 12, 2, 64, (32,), False),                 # wavefronts that have several rows of heads; through the caches
    ("f16", 1030, 28, 4, 128, (16, 24, 24), False),          # two wavefronts a token
    ("f32", 2049, 3, 1, 72, (32,), True),
    ("bf16", 4500, 28, 4, 128, (16, 24, 24), False),         # 41 MB: past the caches
    ("f16", 4500, 28, 4, 128, (64,), True),
    ("f32", 3000, 16, 16, 72, (36,), False),
])
def test_qk_norm_rope_of_many_tokens(bench, dtype, n, H, K, d, sections, interleaved):
    gen, page = _gen(n + H), 16
    pages = -(-n // page) + 2
    x = torch.randn(n, H + 2 * K, d, generator=gen).to(C.TYPES[dtype])
    weight = [(1 + 0.2 * torch.randn(d, generator=gen)).to(C.TYPES[dtype]) for _ in range(2)]
    pos = torch.randint(0, 40000, (n, 3), generator=gen, dtype=torch.int32)
    freq = 1e6 ** (-torch.arange(sum(sections), dtype=torch.float32) / sum(sections))
    slots = torch.randperm(pages * page, generator=gen)[:n]
    kv = [bench.guarded(torch.full((pages, K, page, d), 3.0, dtype=C.TYPES[dtype])) for _ in range(2)]
    q_out, xd = bench.guarded(torch.zeros(n, H, d, dtype=C.TYPES[dtype])), bench.put(x)
    bench.ctx.sttm_qk_norm_rope(xd[:, :H], xd[:, H:H + K], xd[:, H + K:], q_out, cache=bench.lib.PagedCache(*kv), slots=bench.put(slots),
                                q_weight=bench.put(weight[0]), k_weight=bench.put(weight[1]), eps=1e-5,
                                rope=bench.lib.Rope(bench.put(pos), bench.put(freq), sections, interleaved))
    bench.done()
    C.close(q_out, *C.rope_reference(x[:, :H], weight[0], 1e-5, pos, freq, sections, interleaved, C.U[dtype]), what="q")
    k, v = [y.cpu().transpose(1, 2).reshape(pages * page, K, d) for y in kv]
    C.close(k[slots], *C.rope_reference(x[:, H:H + K], weight[1], 1e-5, pos, freq, sections, interleaved, C.U[dtype]), what="cached keys")
    assert torch.equal(v[slots], x[:, H + K:])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots] = False
    assert (k[rest] == 3).all() and (v[rest] == 3).all()


@pytest.mark.parametrize("dtype,B,K,H,d,longest,counts", [
    ("bf16", 1, 4, 28, 128, 16383, False),                   # on both sides of 65,536 slots in all rows
    ("bf16", 1, 4, 28, 128, 16384, True),
    ("f32", 1, 4, 4, 72, 16384, True),
    ("f32", 1, 2, 8, 64, 32767, False),
    ("bf16", 6, 8, 8, 16, 43690, False),                     # ... and of 2,097,152
    ("bf16", 6, 8, 8, 16, 43691, True),
    ("f16", 6, 8, 16, 16, 43691, False),
    ("bf16", 1, 1, 2, 32, 40001, True),                      # more than 256 chunks of each length
    ("f16", 1, 1, 3, 32, 65535, False),
    ("f32", 1, 1, 1, 16, 140000, True),
    ("bf16", 16, 1, 1, 8, 150000, False),
])
def test_paged_attention_on_both_sides_of_its_rules(bench, dtype, B, K, H, d, longest, counts):
    gen, page = _gen(longest + d), 64
    lengths = [longest] + [max(1, longest * (i + 1) // (40 * B)) for i in range(B - 1)]
    need = [-(-n // page) for n in lengths]
    kv = [torch.randn(sum(need), K, page, d, generator=gen).to(C.TYPES[dtype]) for _ in range(2)]
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    free = torch.randperm(sum(need), generator=gen).to(torch.int32)
    for b in range(B):
        table[b, :need[b]] = free[sum(need[:b]):sum(need[:b + 1])]
    q = (torch.randn(B, H, d, generator=gen) * 2).to(C.TYPES[dtype])
    bias = None
    if counts:
        bias = torch.exp(torch.randn(B, K, longest, generator=gen)).ceil().log()
        bias[torch.rand(B, K, longest, generator=gen) < 0.1] = -C.INF
    win, zero, lens = torch.rand(B, K, longest, generator=gen), torch.zeros(B, K, longest), torch.tensor(lengths, dtype=torch.int32)
    want = C.attention_reference(q, *kv, table, lens, page, d ** -0.5, bias, win, zero, dtype)
    got = C.run_attention(bench, q, kv, "pages", table, lens, d ** -0.5, bias, win, zero)
    for name, g, w in zip(("out", "lse", "weights"), got, want):
        C.close(g, *w, what=name)
    alone = C.run_attention(bench, q, kv, "pages", table, lens, d ** -0.5, bias, max_len=longest)   # without weights: the same bits
    assert torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1])


@pytest.mark.parametrize("n,keep", [(2048, 2047), (2049, 1000), (8192, 8191), (8192, 300), (8193, 8192), (12289, 4000)])
@pytest.mark.parametrize("kind", ["spread", "close", "equal"])
def test_cache_evict_on_both_sides_of_its_rules(bench, n, keep, kind):
    """Rows of one workgroup of either size and of several; weights whose first digits tell them apart or do not."""
    gen, K, page = _gen(n), 3, 64
    pages = -(-n // page) + 1
    kv = [torch.randn(pages, K, page, 8, generator=gen).to(torch.bfloat16) for _ in range(2)]
    table = torch.randperm(pages, generator=gen).to(torch.int32)[None].contiguous()
    w = {"spread": torch.randn(1, K, n, generator=gen).mul(2).exp(), "close": 1 + torch.rand(1, K, n, generator=gen) * 1e-3,
         "equal": torch.full((1, K, n), 0.25)}[kind]
    ids = torch.stack([torch.randperm(n, generator=gen) for _ in range(K)])[None].to(torch.int32)
    bias, lens, keeps = torch.randn(1, K, n, generator=gen), torch.tensor([n], dtype=torch.int32), torch.tensor([keep], dtype=torch.int32)
    outs = [torch.zeros_like(w), torch.zeros_like(ids), torch.zeros_like(bias)]
    want = C.evict_reference(*kv, table, lens, page, keeps, None, 4, 64, w, ids, bias, *outs)
    got = C.run_evict(bench, kv, "pages", 8, table, lens, keeps, None, 4, 64, w, ids, bias, *outs)
    for name, g, x in zip(("k", "v", "weights", "ids", "bias", "lengths"), got, want):
        assert torch.equal(g.cpu(), x), name
