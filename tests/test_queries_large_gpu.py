"""The attention of several queries and the sum behind a block on the GPU: at sizes on both sides of every rule that goes by size, past offsets of
32 bits, twice with the same bits, in graphs, side by side, and together."""
import importlib.util
import os

import pytest
import torch

from tests import cache_cases as C
from tests import query_cases as Q
from tests.cache_cases import E, INF, TYPES, U, close
from tests.residual_tests import _norms, _reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def bench(lib):
    return C.Bench(lib, lib.Sttm(0), DEV)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _attend(q, k, v, scale, bias, seen, dtype):
    """Q.attend for many rows at once, on the GPU in 64 bits: q [m, d], k, v [n, d], bias [n] or None, seen bool [m, n] or None."""
    q, k, v = q.double(), k.double(), v.double()
    x, D = (q @ k.T) * scale, (q.abs() @ k.abs().T) * abs(scale)
    if bias is not None:
        x, D = x + bias.double(), D + torch.where(bias == -INF, 0.0, bias).double().abs()
    dead = torch.zeros_like(x, dtype=torch.bool) if seen is None else ~seen
    if bias is not None:
        dead = dead | (bias == -INF)
    x = torch.where(dead, -INF, x)
    D = torch.where(dead, 0.0, D).amax(1, keepdim=True) * (q.shape[1] + 4) * E
    n, none = k.shape[0], dead.all(1)
    lse = torch.logsumexp(x, 1)
    p = torch.where(none[:, None], 0.0, torch.exp(x - torch.where(none, 0.0, lse)[:, None]))
    out = p @ v
    rounded = 0.0 if dtype == "f32" else U[dtype]
    tol = (p @ v.abs()) * (2 * D + (n + 64) * E + rounded) + (2.0 ** -40 * v.abs().sum(0) if dtype == "f16" else 0)
    lse_tol = torch.where(none, 0.0, D[:, 0] + (n + 64) * E + 4 * E * x.amax(1).abs())
    return out, tol + U[dtype] * (1 + 2 ** -6) * out.abs() + Q.LEAST[dtype], lse, lse_tol


CROSS = [
    # dtype, q_heads, kv_heads, d, tokens (None: one each), states, counts
    ("bf16", 28, 4, 128, None, (512, 3, 257), False),              # few rows, one chunk
    ("bf16", 28, 4, 128, None, (513, 70, 0, 300), True),           # few rows, two chunks, most sequences in one of them
    ("f16", 64, 8, 128, None, (8117, 1013, 40, 4000), True),       # chunks of several lengths' ends, a join of 256 lanes a row
    ("f32", 16, 16, 72, (30, 1, 32), (4979, 333, 2000), True),     # few rows: 32 tokens a head
    ("f32", 16, 16, 72, (31, 32, 34), (700, 333, 2000), True),     # many: one more than 32 a segment
    ("bf16", 2, 1, 256, (16,), (3000,), False),                    # rows of 512 bytes
    ("f32", 4, 1, 256, (8, 1), (1500, 2111), False),               # rows of 1024 bytes
    ("bf16", 28, 4, 128, (331,), (9001,), True),                   # many rows, many chunks, a join of a wavefront a row
    ("f16", 10, 5, 200, (140, 200), (1200, 4700), False),
    ("bf16", 6, 2, 64, (2100,), (77,), False),                     # no second launch
    ("f32", 3, 1, 128, (700, 3), (1111, 2500), True),
    ("bf16", 4, 4, 96, tuple([1, 2, 3] * 500), tuple([5, 0, 40] * 500), False),   # a search over many segments
    ("f16", 16, 2, 80, (129, 128, 127), (4095, 4096, 4097), True),
]


def _cross(bench, case, repeats=1):
    dtype, H, K, d, tokens, lengths, counts = case
    gen = _gen(H * d + sum(lengths))
    rows = sum(lengths) + 5
    kv = torch.randn(rows, 2 * K, d, generator=gen).to(TYPES[dtype]).to(DEV)
    offsets, q_offsets = Q.offsets_of(lengths, 2), None if tokens is None else Q.offsets_of(tokens)
    T = len(lengths) if tokens is None else sum(tokens)
    q = (torch.randn(T, H, d, generator=gen) * 2).to(TYPES[dtype]).to(DEV)
    bias = None
    if counts:
        bias = torch.exp(torch.randn(rows, generator=gen)).ceil().log()
        bias[torch.rand(rows, generator=gen) < 0.2] = -INF
        bias = bias.to(DEV)
    st = bench.lib.States(kv[:, :K], kv[:, K:], bench.put(offsets), max(lengths))
    need = bench.lib.sttm_cross_attention_workspace_bytes(st, T, H)
    results = []
    for _ in range(repeats):
        out, lse = bench.guarded(torch.full((T, H, d), 7.0, dtype=TYPES[dtype])), bench.guarded(torch.full((T, H), 7.0))
        bench.ctx.sttm_cross_attention(q, st, out, d ** -0.5, q_offsets=bench.put(q_offsets), key_bias=bias, lse=lse, workspace=bench.workspace(need))
        bench.done()
        results.append((out, lse))
    return q, kv[:, :K], kv[:, K:], offsets, q_offsets, bias, results


@pytest.mark.parametrize("case", CROSS, ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:70])
def test_cross_attention_over_many_states(bench, case):
    dtype, H, K, d, tokens, lengths, counts = case
    q, k, v, offsets, q_offsets, bias, ((out, lse), again) = _cross(bench, case, 2)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])       # (the same bits)
    step = max(1, len(lengths) // 12)
    for b in range(0, len(lengths), step):
        a0, a1 = (b, b + 1) if q_offsets is None else (int(q_offsets[b]), int(q_offsets[b + 1]))
        k0, k1 = int(offsets[b]), int(offsets[b + 1])
        for h in range(H):
            g = h // (H // K)
            want = _attend(q[a0:a1, h], k[k0:k1, g], v[k0:k1, g], d ** -0.5, None if bias is None else bias[k0:k1], None, dtype) if k1 > k0 else None
            if want is None:
                assert (out[a0:a1, h] == 0).all() and (lse[a0:a1, h] == -INF).all()
                continue
            close(out[a0:a1, h], want[0].cpu(), want[1].cpu(), what=f"out {b} {h}")
            close(lse[a0:a1, h], want[2].cpu(), want[3].cpu(), what=f"lse {b} {h}")


SHARED = [
    # dtype, q_heads, kv_heads, d, page, prefixes, sequences before each group, own, tokens (None: one each), counts
    ("bf16", 28, 4, 128, 16, (9000,), (0, 32), tuple(range(1, 417, 13)), None, True),          # a step of many answers
    ("f16", 64, 8, 128, 32, (901, 4000, 2100), (0, 1, 4, 7), (700, 1, 300, 33, 64, 65, 5), None, False),
    ("bf16", 28, 4, 128, 16, (1200, 2300), (0, 3, 5), (60, 211, 13, 100, 128), (60, 211, 13, 100, 128), True),
    ("f32", 16, 16, 72, 16, (1500,), (1, 3), (900, 40, 41), (50, 1, 40), True),
    ("bf16", 3, 1, 256, 8, (700,), (0, 2), (600, 200), (40, 2), False),
    ("f16", 8, 2, 64, 64, None, None, (3000, 40), (700, 40), False),                                # a prompt in several calls: causal, own past
    ("bf16", 14, 2, 64, 16, (40, 0), (0, 2, 2), (1500, 2000), (1, 1), True),
]


@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:70])
def test_shared_attention_over_many_slots(bench, case):
    dtype, H, K, d, page, lengths, groups, own, tokens, counts = case
    gen, n = _gen(H * d + sum(own)), len(lengths or ())
    kv, table = C.pool(gen, dtype, K, d, page, (lengths or ()) + own, order="pages")
    kv = [x.to(DEV) for x in kv]
    cache = bench.lib.PagedCache(*kv)
    T = len(own) if tokens is None else sum(tokens)
    q_offsets = Q.offsets_of(tokens or (1,) * len(own))
    q = (torch.randn(T, H, d, generator=gen) * 2).to(TYPES[dtype]).to(DEV)
    pre = None if lengths is None else bench.lib.Sequences(table[:n].contiguous().to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), max(lengths))
    seqs = bench.lib.Sequences(table[n:].contiguous().to(DEV), torch.tensor(own, dtype=torch.int32, device=DEV), max(own))
    bias = None
    if counts:
        bias = torch.exp(torch.randn(n, K, max(lengths), generator=gen)).ceil().log()
        bias[torch.rand(bias.shape, generator=gen) < 0.2] = -INF
        bias = bias.to(DEV)
    need, results = bench.lib.sttm_shared_attention_workspace_bytes(cache, pre, seqs, T, H), []
    for _ in range(2):
        out, lse = bench.guarded(torch.full((T, H, d), 7.0, dtype=TYPES[dtype])), bench.guarded(torch.full((T, H), 7.0))
        bench.ctx.sttm_shared_attention(q, cache, pre, None if groups is None else torch.tensor(groups, dtype=torch.int32, device=DEV), seqs, out, d ** -0.5,
                                        q_offsets=None if tokens is None else q_offsets.to(DEV), prefix_bias=bias, lse=lse, workspace=bench.workspace(need))
        bench.done()
        results.append((out, lse))
    (out, lse), again = results
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    for b, m in enumerate(tokens or (1,) * len(own)):
        a0, a1 = int(q_offsets[b]), int(q_offsets[b + 1])
        parts = [(table[n + b], own[b], None)]
        g = [g for g in range(n) if groups[g] <= b < groups[g + 1]]
        if g:
            parts.insert(0, (table[g[0]], lengths[g[0]], None if bias is None else bias[g[0]]))
        rows = [torch.tensor([int(t[i // page]) * page + i % page for i in range(s)], device=DEV, dtype=torch.int64) for t, s, _ in parts]
        at = torch.cat(rows)
        add = torch.cat([torch.zeros(K, s, device=DEV) if c is None else c[:, :s] for _, s, c in parts], 1)
        seen = torch.ones(m, len(at), dtype=torch.bool, device=DEV)
        seen[:, len(at) - own[b]:] = torch.arange(own[b], device=DEV) < (own[b] - m + 1 + torch.arange(m, device=DEV))[:, None]
        for h in range(H):
            c = h // (H // K)
            k, v = (x[at // page, c, at % page] for x in kv)
            want = _attend(q[a0:a1, h], k, v, d ** -0.5, add[c], seen, dtype)
            close(out[a0:a1, h], want[0].cpu(), want[1].cpu(), what=f"out {b} {h}")
            close(lse[a0:a1, h], want[2].cpu(), want[3].cpu(), what=f"lse {b} {h}")


@pytest.mark.parametrize("dtype,n,D,gate", [("bf16", 5000, 3584, "row"), ("f32", 4099, 1152, "one"), ("f16", 3500, 4160, "channel"), ("f32", 3100, 16384, "none"),
                                            ("bf16", 70000, 64, "full")])
def test_residual_norm_of_many_rows(bench, dtype, n, D, gate):
    """More rows than workgroups, rows of one and of several loads a lane."""
    gen, t = _gen(D + n), TYPES[dtype]
    x, y = ((torch.randn(n, D, generator=gen) * 2).to(t) for _ in range(2))
    shape = {"none": None, "one": (1, 1), "row": (n, 1), "channel": (1, D), "full": (n, D)}[gate]
    g = None if shape is None else torch.randn(shape, generator=gen).to(t)
    post, pre = _norms("rms", D, gen, dtype), _norms("layer", D, gen, dtype)
    norm = lambda z, kind: bench.lib.Norm(kind, bench.put(z[1]), bench.put(z[2]), z[3])   # noqa: E731
    r, h = bench.guarded(torch.zeros(n, D, dtype=t)), bench.guarded(torch.zeros(n, D, dtype=t))
    bench.ctx.sttm_residual_norm(bench.put(x), bench.put(y), r, h, post=norm(post, bench.lib.STTM_NORM_RMS), pre=norm(pre, bench.lib.STTM_NORM_LAYER),
                                 gate=bench.put(g), gate_tanh=True)
    bench.done()
    some = torch.cat([torch.arange(0, n, max(1, n // 300)), torch.arange(n - 20, n)])
    part = None if g is None else g[some] if g.shape[0] == n else g
    want = _reference(x[some], y[some], part, True, 1.0, post, pre, dtype)
    close(r[some.to(DEV)], *want[0], what="r")
    close(h[some.to(DEV)], *want[1], what="h")


# -- the largest calls -------------------------------------------------------------------------------------------------

def test_as_many_sequences_as_there_may_be(bench):
    """65,535 sequences of one state, and of one own slot behind a prefix that none of them has: results are the values themselves."""
    lib, n, d = bench.lib, 65535, 8
    gen = torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.randn(n, 1, d, device=DEV, generator=gen).to(torch.bfloat16) for _ in range(3))
    st = lib.States(k, v, torch.arange(n + 1, device=DEV), 1)
    out, lse = torch.zeros_like(q), torch.zeros(n, 1, device=DEV)
    bench.ctx.sttm_cross_attention(q, st, out, 0.5, lse=lse, workspace=bench.workspace(lib.sttm_cross_attention_workspace_bytes(st, n, 1)))
    bench.done()
    score = (q.double() * k.double()).sum(2) * 0.5
    assert torch.equal(out, v) and float((lse.double() - score).abs().max()) < 1e-4
    page, pages = 8, n // 8 + 1
    pool = [torch.zeros(pages * page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for x, y in zip(pool, (k, v)):
        x[::page] = y[:pages, 0]
    cache = lib.PagedCache(*[x.view(pages, 1, page, d) for x in pool])
    own = lib.Sequences((torch.arange(n, device=DEV, dtype=torch.int32) % pages)[:, None].contiguous(), torch.ones(n, dtype=torch.int32, device=DEV), 1)
    pre = lib.Sequences(torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.tensor([8], dtype=torch.int32, device=DEV), 8)
    groups, out = torch.tensor([n, n], dtype=torch.int32, device=DEV), torch.zeros_like(q)
    bench.ctx.sttm_shared_attention(q, cache, pre, groups, own, out, 0.5,
                                    workspace=bench.workspace(lib.sttm_shared_attention_workspace_bytes(cache, pre, own, n, 1)))
    bench.done()
    assert torch.equal(out, v[torch.arange(n, device=DEV) % pages])


def test_as_many_tokens_and_rows_as_there_may_be(bench):
    lib, n, d = bench.lib, 1 << 22, 8
    gen = torch.Generator(device=DEV).manual_seed(2)
    q = torch.randn(n, 1, d, device=DEV, generator=gen).to(torch.float16)
    k, v = (torch.randn(300, 1, d, device=DEV, generator=gen).to(torch.float16) for _ in range(2))
    st, out = lib.States(k, v, torch.tensor([0, 300], device=DEV)), torch.zeros_like(q)
    bench.ctx.sttm_cross_attention(q, st, out, 0.3, q_offsets=torch.tensor([0, n], device=DEV),
                                   workspace=bench.workspace(lib.sttm_cross_attention_workspace_bytes(st, n, 1)))
    bench.done()
    some = torch.cat([torch.arange(0, n, 9973, device=DEV), torch.arange(n - 200, n, device=DEV)])
    want = _attend(q[some, 0], k[:, 0], v[:, 0], 0.3, None, None, "f16")
    close(out[some, 0], want[0].cpu(), want[1].cpu(), what="out")
    x = torch.randn(1 << 25, 8, device=DEV, generator=gen).to(torch.bfloat16)
    r = torch.zeros_like(x)
    bench.ctx.sttm_residual_norm(x, None, r, None, scale=2.0)
    bench.done()
    assert torch.equal(r, x * 2)


# -- offsets beyond 32 bits --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [1, 70])
def test_states_further_apart_than_four_gigabytes(bench, tokens):
    """Rows of 4 MB stride: keys of one sequence and of the next beyond 2^31 elements' bytes from the first, heads 2^32 bytes apart."""
    n, d, stride, apart = 1100, 64, 1 << 21, (1 << 31) + 4096
    gen = _gen(4)
    raw = torch.zeros(apart + n * stride, dtype=torch.bfloat16, device=DEV)
    k = raw.as_strided((n, 2, d), (stride, apart, 1))
    v = raw[d:].as_strided((n, 2, d), (stride, apart, 1))
    data = [torch.randn(n, 2, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2)]
    k.copy_(data[0])
    v.copy_(data[1])
    offsets, q_offsets = torch.tensor([0, 20, n]), Q.offsets_of((tokens, tokens))
    st = bench.lib.States(k, v, bench.put(offsets), n)
    q = torch.randn(2 * tokens, 4, d, generator=gen).to(torch.bfloat16).to(DEV)
    out = bench.guarded(torch.zeros(2 * tokens, 4, d, dtype=torch.bfloat16))
    bench.ctx.sttm_cross_attention(q, st, out, 0.125, q_offsets=bench.put(q_offsets),
                                   workspace=bench.workspace(bench.lib.sttm_cross_attention_workspace_bytes(st, 2 * tokens, 4)))
    bench.done()
    for b, (k0, k1) in enumerate(((0, 20), (20, n))):
        for h in range(4):
            want = _attend(q[b * tokens:(b + 1) * tokens, h], data[0][k0:k1, h // 2], data[1][k0:k1, h // 2], 0.125, None, None, "bf16")
            close(out[b * tokens:(b + 1) * tokens, h], want[0].cpu(), want[1].cpu(), what=f"out {b} {h}")


@pytest.mark.parametrize("tokens", [1, 40])
def test_a_pool_of_more_than_four_gigabytes_behind_several_queries(bench, tokens):
    lib, gen = bench.lib, _gen(8)
    K, d, page, stride = 2, 64, 16, (1 << 32) + 4096
    view = [torch.zeros(2 * stride + (1 << 20), dtype=torch.float16, device=DEV).as_strided((3, K, page, d), (stride, page * d, d, 1)) for _ in range(2)]
    data = [torch.randn(3, K, page, d, generator=gen).half() for _ in range(2)]
    for x, y in zip(view, data):
        x.copy_(y.to(DEV))
    cache = lib.PagedCache(*view)
    pre = (torch.tensor([[2, 0]], dtype=torch.int32), torch.tensor([30], dtype=torch.int32))
    own = (torch.tensor([[1, 2, 0]], dtype=torch.int32), torch.tensor([44], dtype=torch.int32))
    q = torch.randn(tokens, 4, d, generator=gen).half()
    cuts, q_offsets = torch.tensor([0, 1], dtype=torch.int32), Q.offsets_of((tokens,))
    seven = torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0)
    want = Q.shared_reference(q, q_offsets, *data, page, pre, cuts, own, 0.125, None, None, *seven, "f16")
    p, s = (lib.Sequences(bench.put(x[0]), bench.put(x[1])) for x in (pre, own))
    out = bench.guarded(torch.full_like(q, 7.0))
    bench.ctx.sttm_shared_attention(bench.put(q), cache, p, bench.put(cuts), s, out, 0.125, q_offsets=bench.put(q_offsets),
                                    workspace=bench.workspace(lib.sttm_shared_attention_workspace_bytes(cache, p, s, tokens, 4)))
    bench.done()
    close(out, *want[0], what="out")


# -- graphs and streams ------------------------------------------------------------------------------------------------

class _Layer:
    """A layer's calls one behind the other: cross-attention, the gated sum behind it, attention behind a shared prefix; buffers of its own."""

    def __init__(self, lib, seed):
        gen = _gen(seed)
        K, H, d, page, B = 2, 8, 128, 16, 5
        r = lambda *s: torch.randn(*s, generator=gen).to(torch.bfloat16).to(DEV)   # noqa: E731
        self.lib, self.q, self.states = lib, r(B, H, d), r(1700, 2 * K, d)
        offsets = Q.offsets_of((700, 100, 0, 800, 100)).to(DEV)
        self.st = lib.States(self.states[:, :K], self.states[:, K:], offsets, 800)
        self.counts = torch.rand(1700, generator=gen).to(DEV)
        kv, table = C.pool(gen, "bf16", K, d, page, (900, 60, 5, 33, 80, 1), order="pages")
        self.kv = [x.to(DEV) for x in kv]
        self.cache = lib.PagedCache(*self.kv)
        self.pre = lib.Sequences(table[:1].contiguous().to(DEV), torch.tensor([900], dtype=torch.int32, device=DEV), 900)
        self.seqs = lib.Sequences(table[1:].contiguous().to(DEV), torch.tensor([60, 5, 33, 80, 1], dtype=torch.int32, device=DEV), 80)
        self.groups = torch.tensor([0, 5], dtype=torch.int32, device=DEV)
        self.x, self.gate = r(B, H * d), r(1, 1)
        self.norm = lib.Norm(lib.STTM_NORM_RMS, r(H * d))
        self.out, self.out2 = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.lse, self.r, self.h = torch.zeros(B, H, device=DEV), torch.zeros_like(self.x), torch.zeros_like(self.x)
        need = max(lib.sttm_cross_attention_workspace_bytes(self.st, B, H), lib.sttm_shared_attention_workspace_bytes(self.cache, self.pre, self.seqs, B, H))
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)

    def step(self, ctx):
        ctx.sttm_cross_attention(self.q, self.st, self.out, 0.1, key_bias=self.counts, workspace=self.ws)
        ctx.sttm_residual_norm(self.x, self.out.view(5, -1), self.r, self.h, post=self.norm, pre=self.norm, gate=self.gate, gate_tanh=True)
        ctx.sttm_shared_attention(self.h.view_as(self.q), self.cache, self.pre, self.groups, self.seqs, self.out2, 0.1, lse=self.lse, workspace=self.ws)

    def result(self):
        return [x.clone() for x in (self.out, self.r, self.h, self.out2, self.lse)]

    def reset(self):
        for x in (self.out, self.r, self.h, self.out2, self.lse):
            x.zero_()


def test_two_graphs_of_a_layer_on_streams_of_their_own(lib):
    """Captured on two streams with a workspace each, replayed in turn, at once, with eager calls and synchronisation between: every replay
    gives what the eager calls give."""
    ctx, layers, graphs, streams, want = lib.Sttm(0), [_Layer(lib, 1), _Layer(lib, 2)], [], [torch.cuda.Stream(), torch.cuda.Stream()], []
    for layer in layers:
        layer.step(ctx)
        torch.cuda.synchronize()
        want.append(layer.result())
        assert all(torch.isfinite(x).all() for x in want[-1][:4])
    for layer, stream in zip(layers, streams):
        with torch.cuda.stream(stream):
            own = lib.Sttm(0)
            layer.step(own)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                layer.step(own)
            graphs.append((graph, own))
    eager = _Layer(lib, 1)
    for _ in range(4):
        torch.cuda.synchronize()
        for layer in layers:
            layer.reset()
        torch.randn(1 << 20, device=DEV).sum().item()
        torch.cuda.synchronize()
        for (graph, _), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager.step(ctx)
        torch.cuda.synchronize()
        for layer, expected in zip(layers + [eager], want + [want[0]]):
            for a, b in zip(layer.result(), expected):
                assert torch.equal(a, b)
        eager.reset()


def test_lengths_that_change_between_replays(lib):
    """Offsets, lengths, tables and biases are read when a graph runs, not when it is captured."""
    ctx, layer, side = lib.Sttm(0), _Layer(lib, 3), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        own = lib.Sttm(0)
        layer.step(own)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.step(own)
    for lengths, prefix in (((1, 2, 3, 4, 5), 31), ((700, 100, 0, 800, 100), 900), ((0, 0, 0, 0, 799), 0)):
        torch.cuda.synchronize()
        layer.st.offsets.copy_(Q.offsets_of(lengths))
        layer.pre.lengths.fill_(prefix)
        layer.reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = layer.result()
        layer.reset()
        layer.step(ctx)
        torch.cuda.synchronize()
        for a, b in zip(got, layer.result()):
            assert torch.equal(a, b)


def test_questions_about_one_video_run_the_operators_together():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "questions_about_one_video.py")
    spec = importlib.util.spec_from_file_location("questions_about_one_video", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)                       # (finds the other example beside it)
    from paper_2507_07990_amd import workloads as wl
    r = example.run(wl.small_variant(wl.CONFIGS[1], T=6, D=1792), keep=0.5, questions=(5, 9, 2), steps=4)
    assert r["kept"] <= r["video_tokens"] // 2 and r["cached"] == [5 + 4, 9 + 4, 2 + 4] and r["answers"] == 12 and r["finite"]
