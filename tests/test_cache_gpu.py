"""The operators on a paged cache on the GPU, against the definitions in 64 bits."""
import pytest
import torch

from tests import cache_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bench(lib):
    return C.Bench(lib, lib.Sttm(0), "cuda:0")


from tests.cache_tests import *  # noqa: E402,F401,F403  -- the tests that run on host threads too


@pytest.mark.parametrize("n,keep,kind", [(20001, 7000, "spread"), (50003, 25000, "ties"), (70001, 69000, "spread"), (66000, 20000, "equal")])
def test_cache_evict_of_long_rows(bench, n, keep, kind):
    """Rows whose keys fill a wavefront's registers, and rows too long for them."""
    gen = torch.Generator().manual_seed(n)
    kv, table = C.pool(gen, "bf16", 1, 8, 1024, (0,), spare=-(-n // 1024) + 1)
    table = torch.randperm(kv[0].shape[0], generator=gen).to(torch.int32)[None].contiguous()
    kv = [torch.randn(x.shape, generator=gen).to(x.dtype) for x in kv]
    w = torch.randn(1, 1, n, generator=gen).mul(3).exp()
    if kind == "ties":
        w = torch.randint(0, 2, (1, 1, n), generator=gen).float()
    if kind == "equal":
        w = torch.zeros(1, 1, n)
    ids = torch.randperm(n, generator=gen).to(torch.int32).view(1, 1, n)
    lens, keeps = torch.tensor([n], dtype=torch.int32), torch.tensor([keep], dtype=torch.int32)
    outs = [torch.zeros_like(w), torch.zeros_like(ids), None]
    want = C.evict_reference(*kv, table, lens, 1024, keeps, None, 4, 300, w, ids, None, *outs)
    got = C.run_evict(bench, kv, "pages", 8, table, lens, keeps, None, 4, 300, w, ids, None, *outs)
    for name, g, x in zip(("k", "v", "weights", "ids", "bias", "lengths"), got, want):
        assert x is None or torch.equal(g.cpu(), x), name


@pytest.mark.parametrize("dtype,lengths,weights", [("bf16", (9000, 1, 4097), True), ("f16", (20000,), True), ("f32", (2500, 3000), False)])
def test_paged_attention_over_long_sequences(bench, dtype, lengths, weights):
    """Many chunks, joined; the same bits on every call."""
    gen = torch.Generator().manual_seed(sum(lengths))
    H, K, d, page, B = 6, 2, 64, 32, len(lengths)
    need = [-(-n // page) for n in lengths]
    kv = [torch.randn(sum(need), K, page, d, generator=gen).to(C.TYPES[dtype]) for _ in range(2)]
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    free = torch.randperm(sum(need), generator=gen).to(torch.int32)
    for b in range(B):
        table[b, :need[b]] = free[sum(need[:b]):sum(need[:b + 1])]
    q = (torch.randn(B, H, d, generator=gen) * 2).to(C.TYPES[dtype])
    cap = max(lengths)
    win = torch.rand(B, K, cap, generator=gen) if weights else None
    wout = torch.zeros(B, K, cap) if weights else None
    lens = torch.tensor(lengths, dtype=torch.int32)
    want = C.attention_reference(q, *kv, table, lens, page, 0.125, None, win, wout, dtype)
    got = C.run_attention(bench, q, kv, "pages", table, lens, 0.125, None, win, wout)
    again = C.run_attention(bench, q, kv, "pages", table, lens, 0.125, None, win, wout)
    for name, g, a, w in zip(("out", "lse", "weights"), got, again, want):
        if w[0] is not None:
            C.close(g, *w, what=name)
            assert torch.equal(g, a), name


def test_a_pool_of_more_than_four_gigabytes(bench):
    """Rows whose addresses lie beyond 32 bits from the pool's, through all three operators."""
    lib, ctx, gen = bench.lib, bench.ctx, torch.Generator().manual_seed(8)
    K, d, page, n, stride = 2, 64, 16, 44, (1 << 32) + 4096
    big = [torch.empty(2 * stride + (1 << 20), dtype=torch.float16, device="cuda:0") for _ in range(2)]
    view = [x.as_strided((3, K, page, d), (stride, page * d, d, 1)) for x in big]
    for x in view:
        x.zero_()
    cache = lib.PagedCache(*view)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    seqs = lib.Sequences(table.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), n)
    x = torch.randn(n, 4 + 2 * K, d, generator=gen).half()
    i = torch.arange(n)
    slots = table[0].long()[i // page] * page + i % page
    qo = torch.zeros(n, 4, d, dtype=torch.float16, device="cuda:0")
    xd = x.cuda()
    ctx.sttm_qk_norm_rope(xd[:, :4], xd[:, 4:4 + K], xd[:, 4 + K:], qo, cache=cache, slots=slots.cuda())
    torch.cuda.synchronize()
    host = [v.cpu() for v in view]
    assert torch.equal(host[0][slots // page, :, slots % page], x[:, 4:4 + K]) and torch.equal(host[1][slots // page, :, slots % page], x[:, 4 + K:])
    q, w0 = torch.randn(1, 4, d, generator=gen).half(), torch.zeros(1, K, n)
    out, w = torch.zeros(1, 4, d, dtype=torch.float16, device="cuda:0"), torch.zeros(1, K, n, device="cuda:0")
    ws = bench.workspace(max(lib.sttm_paged_attention_workspace_bytes(cache, seqs, 4, True), lib.sttm_cache_evict_workspace_bytes(cache, seqs)))
    ctx.sttm_paged_attention(q.cuda(), cache, seqs, out, 0.125, weights_out=w, workspace=ws)
    want = C.attention_reference(q, *host, table, torch.tensor([n]), page, 0.125, None, None, w0, "f16")
    C.close(out, *want[0], what="out")
    C.close(w, *want[2], what="weights")
    keep, new, ids = torch.tensor([20], dtype=torch.int32), torch.zeros(1, dtype=torch.int32, device="cuda:0"), torch.zeros(1, K, n, dtype=torch.int32)
    wr = torch.rand(1, K, n, generator=gen)
    wo, io = torch.zeros(1, K, n, device="cuda:0"), ids.cuda()
    want = C.evict_reference(*host, table, torch.tensor([n]), page, keep, None, 0, 0, wr, None, None, torch.zeros_like(wr), ids, None)
    ctx.sttm_cache_evict(cache, seqs, keep.cuda(), new, wr.cuda(), wo, None, io, workspace=ws)
    bench.done()
    assert torch.equal(view[0].cpu(), want[0]) and torch.equal(view[1].cpu(), want[1]) and torch.equal(io.cpu(), want[3])


def test_a_step_in_a_graph_on_another_stream(lib):
    """Rotation, cache write, attention and eviction captured on a stream of their own: every replay gives what the eager calls
    give, with other work and synchronisation in between."""
    side = torch.cuda.Stream()
    gen = torch.Generator().manual_seed(9)
    K, H, d, page, B, n = 2, 8, 128, 16, 3, 200
    dev = "cuda:0"
    kv = [torch.randn(64, K, page, d, generator=gen).to(torch.bfloat16) for _ in range(2)]
    table = torch.randperm(64, generator=gen)[:3 * 14].view(3, 14).to(torch.int32)
    lens = torch.tensor([n, 131, 64], dtype=torch.int32)
    x = torch.randn(B, H + 2 * K, d, generator=gen).to(torch.bfloat16)
    at = lens.long() - 1
    slots = table[torch.arange(B), at // page].long() * page + at % page
    weights = torch.rand(B, K, n, generator=gen)

    class State:
        def __init__(self):
            self.kv = [y.to(dev) for y in kv]
            self.cache = lib.PagedCache(*self.kv)
            self.lens, self.new = lens.to(dev), torch.zeros(B, dtype=torch.int32, device=dev)
            self.seqs = lib.Sequences(table.to(dev), self.lens, n)
            self.x, self.q = x.to(dev), torch.zeros(B, H, d, dtype=torch.bfloat16, device=dev)
            self.rope = lib.Rope(lens.to(dev), torch.linspace(1, 0.001, 64, device=dev))
            self.slots, self.out = slots.to(dev), torch.zeros(B, H, d, dtype=torch.bfloat16, device=dev)
            self.win, self.w, self.w2 = weights.to(dev), torch.zeros(B, K, n, device=dev), torch.zeros(B, K, n, device=dev)
            self.ids = torch.zeros(B, K, n, dtype=torch.int32, device=dev)
            self.keep = (lens // 2).to(torch.int32).to(dev)
            self.ws = torch.full((max(lib.sttm_paged_attention_workspace_bytes(self.cache, self.seqs, H, True),
                                      lib.sttm_cache_evict_workspace_bytes(self.cache, self.seqs)),), 255, dtype=torch.uint8, device=dev)

        def reset(self):
            for a, y in zip(self.kv, kv):
                a.copy_(y)
            for y in (self.out, self.w, self.w2, self.ids, self.new):
                y.zero_()

        def step(self, ctx):
            ctx.sttm_qk_norm_rope(self.x[:, :H], self.x[:, H:H + K], self.x[:, H + K:], self.q, cache=self.cache, slots=self.slots, rope=self.rope)
            ctx.sttm_paged_attention(self.q, self.cache, self.seqs, self.out, d ** -0.5, weights_in=self.win, weights_out=self.w, workspace=self.ws)
            ctx.sttm_cache_evict(self.cache, self.seqs, self.keep, self.new, self.w, self.w2, None, self.ids, sink=1, recent=5, workspace=self.ws)

        def result(self):
            return [y.clone() for y in (*self.kv, self.q, self.out, self.w, self.w2, self.ids, self.new)]

    eager = State()
    eager.step(lib.Sttm(0))
    want = eager.result()
    s = State()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx = lib.Sttm(0)
        s.step(ctx)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.step(ctx)
    for _ in range(3):
        torch.cuda.synchronize()
        s.reset()
        torch.randn(1 << 20, device=dev).sum().item()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, y in zip(s.result(), want):
            assert torch.equal(a, y)


def test_the_example_runs_the_operators_together():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_from_reduced_video.py")
    spec = importlib.util.spec_from_file_location("answer_from_reduced_video", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    from paper_2507_07990_amd import workloads as wl
    r = example.run(wl.small_variant(wl.CONFIGS[1], T=6, D=1792), keep=0.5, steps=5, cache_keep=0.5)
    assert r["kept"] <= r["video_tokens"] // 2 and r["cached"] == r["kept"] + 5 and r["steps"] == 10 and r["finite"]
    assert r["cached_after"] == r["cached"] // 2 + 5 and r["similarity"] > 0.5
