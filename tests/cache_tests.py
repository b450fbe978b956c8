"""Tests of the operators on a paged cache that run on the GPU (test_cache_gpu.py) and on host threads (test_cache_cpu.py):
`bench` is the context under test."""
import math

import pytest
import torch

from tests import cache_cases as C
from tests.cache_cases import INF, TYPES, U, close


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# -- norm and rotation -------------------------------------------------------------------------------------------------

ROPE = [
    # dtype, n, q_heads, kv_heads, d, norm, sections, positions, interleaved, cache order, page
    ("bf16", 1, 28, 4, 128, True, (64,), "int", False, "pages", 16),      # one token
    ("bf16", 5, 7, 1, 128, True, (16, 24, 24), "grid", False, "slots", 8),
    ("f16", 3, 2, 2, 80, False, (40,), "float", False, "padded", 16),
    ("f32", 7, 3, 3, 72, True, (32,), "float", True, "pages", 8),         # 8 channels stay
    ("f32", 2, 10, 5, 256, True, (20, 0, 12), "grid", False, "pages", 32),
    ("f16", 4, 1, 1, 8, True, (4,), "int", True, "pages", 8),             # a head of one unit
    ("bf16", 3, 9, 3, 40, True, (20,), "int", False, "slots", 8),
    ("bf16", 2, 2, 1, 64, True, (), "int", False, "pages", 8),            # no rotation
    ("f32", 3, 5, 1, 24, False, (), "int", False, "pages", 8),            # nothing but copies
    ("bf16", 70, 1, 1, 248, True, (4, 4, 4), "grid", True, "pages", 1024),
]


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
@pytest.mark.parametrize("form", ["projection", "in_place"])
def test_qk_norm_rope(bench, case, form):
    dtype, n, H, K, d, norm, sections, kind, interleaved, order, page = case
    gen = _gen(n * d + H)
    kv, table = C.pool(gen, dtype, K, d, page, [0], order=order, spare=-(-(n + 3) // page) + 1)
    pages = kv[0].shape[0]
    slots = torch.randperm(pages * page, generator=gen)[:n]
    if n > 2:
        slots[1], slots[2] = -1, pages * page           # no slots of the pool: skipped
    x = torch.randn(n, (H + 2 * K) * d + 16, generator=gen).to(TYPES[dtype])
    weight = [(1 + 0.2 * torch.randn(d, generator=gen)).to(TYPES[dtype]) if norm else None for _ in range(2)]
    pos = {"int": torch.randint(0, 50000, (n, 1), generator=gen, dtype=torch.int32),
           "float": torch.rand(n, 2, generator=gen) * 30000,
           "grid": torch.randint(0, 600, (n, 4), generator=gen, dtype=torch.int32)}[kind]
    freq = 1e6 ** (-torch.arange(sum(sections), dtype=torch.float32) / max(1, sum(sections)))

    def split(t):
        t = t[:, :(H + 2 * K) * d].view(n, H + 2 * K, d) if t.is_contiguous() and t.shape[1] == (H + 2 * K) * d else t[:, :-16].unflatten(1, (H + 2 * K, d))
        return t[:, :H], t[:, H:H + K], t[:, H + K:]

    want = [C.rope_reference(y, w, 1e-5, pos, freq, sections, interleaved, U[dtype]) for y, w in zip(split(x), weight)]
    dev = [bench.guarded(y) for y in kv]
    cache = bench.lib.PagedCache(*C.cache_views(dev, order, d))
    xd = bench.guarded(x)
    q, k, v = split(xd)
    if form == "in_place":
        q_out, k_out = q, k
    else:
        q_out, k_out = bench.guarded(torch.full((n, H, d), 3.0, dtype=TYPES[dtype])), None
    rope = bench.lib.Rope(bench.put(pos), bench.put(freq), sections, interleaved) if sections else None
    bench.ctx.sttm_qk_norm_rope(q, k, v, q_out, k_out=k_out, cache=cache, slots=bench.put(slots), q_weight=bench.put(weight[0]),
                                k_weight=bench.put(weight[1]), eps=1e-5, rope=rope)
    bench.done()
    close(q_out, *want[0], what="q")
    if k_out is not None:
        close(k_out, *want[1], what="k")
    assert torch.equal(xd[:, -16:].cpu(), x[:, -16:]), "the padding of the rows was overwritten"
    got = [y.cpu() for y in C.cache_views(dev, order, d)]
    used = torch.zeros(pages, page, dtype=torch.bool)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            used[s // page, s % page] = True
            close(got[0][s // page, :, s % page], want[1][0][i], want[1][1][i], "cached key")
            assert torch.equal(got[1][s // page, :, s % page], split(x)[2][i]), "cached value"
    for y in got:
        assert torch.isnan(y.transpose(1, 2)[~used]).all(), "a slot that no row names was written"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_qk_norm_rope_without_a_cache(bench, dtype):
    """Queries and keys alone, into buffers of their own; a norm for one of the two."""
    gen, n, H, K, d = _gen(4), 6, 5, 2, 48
    q, k = (torch.randn(n, h, d, generator=gen).to(TYPES[dtype]) for h in (H, K))
    w = (1 + 0.2 * torch.randn(d, generator=gen)).to(TYPES[dtype])
    pos, freq = torch.randint(0, 900, (n,), generator=gen, dtype=torch.int32), torch.linspace(1.0, 0.01, d // 2)
    qo, ko = bench.guarded(torch.zeros_like(q)), bench.guarded(torch.zeros_like(k))
    bench.ctx.sttm_qk_norm_rope(bench.put(q), bench.put(k), None, qo, k_out=ko, k_weight=bench.put(w), eps=1e-5,
                                rope=bench.lib.Rope(bench.put(pos), bench.put(freq)))
    bench.done()
    close(qo, *C.rope_reference(q, None, 1e-5, pos[:, None], freq, (d // 2,), False, U[dtype]), what="q")
    close(ko, *C.rope_reference(k, w, 1e-5, pos[:, None], freq, (d // 2,), False, U[dtype]), what="k")


def test_qk_norm_rope_of_rows_that_are_not_finite(bench):
    """An infinity or NaN in one head stays in that head; a row of zeros stays zero."""
    gen = _gen(3)
    x = torch.randn(4, 3, 16, generator=gen)
    x[0, 0, 3], x[1, 1, 5], x[2, 2] = INF, math.nan, 0.0
    w = torch.ones(16)
    pos = torch.arange(4, dtype=torch.int32)
    out = bench.guarded(torch.zeros_like(x))
    k = bench.put(torch.zeros(4, 1, 16))
    freq = torch.ones(8)
    bench.ctx.sttm_qk_norm_rope(bench.put(x), k, None, out, q_weight=bench.put(w), eps=1e-6, rope=bench.lib.Rope(bench.put(pos), bench.put(freq)))
    bench.done()
    got = out.cpu()
    assert torch.isnan(got[0, 0]).any() and torch.isnan(got[1, 1]).all() and (got[2, 2] == 0).all()
    rest = torch.ones(4, 3, dtype=torch.bool)
    rest[0, 0] = rest[1, 1] = False
    assert torch.isfinite(got[rest]).all()


# -- attention ---------------------------------------------------------------------------------------------------------

ATTENTION = [
    # dtype, q_heads, kv_heads, d, page, lengths, order, bias, weights
    ("bf16", 7, 1, 128, 16, (1,), "pages", "", False),
    ("bf16", 14, 2, 128, 16, (33, 0, 300), "pages", "", True),
    ("f16", 4, 2, 80, 8, (31, 32, 129), "slots", "", True),
    ("f32", 3, 3, 72, 16, (5, 160), "pages", "counts", True),
    ("f32", 2, 1, 256, 32, (17, 50), "padded", "", True),
    ("bf16", 2, 2, 256, 8, (9, 140), "pages", "counts", False),
    ("f16", 1, 1, 8, 8, (1, 257), "pages", "counts", True),
    ("bf16", 17, 1, 64, 64, (70, 3), "slots", "counts", True),      # a second tile of heads with one head in it
    ("f16", 33, 1, 40, 16, (40,), "pages", "", True),
    ("f32", 5, 5, 24, 1024, (0, 0), "pages", "", True),             # nothing cached
    ("bf16", 8, 4, 96, 8, (260, 127, 128, 1), "pages", "lowest", True),
    ("f32", 4, 2, 136, 8, (67,), "slots", "empty", True),
    ("bf16", 3, 1, 168, 8, (45,), "pages", "empty", False),
    ("f16", 2, 1, 32, 16, (129,), "padded", "huge", True),
    ("f32", 6, 2, 72, 16, (33, 90), "pages", "counts", True),      # fp32 with groups
    ("f32", 3, 1, 256, 8, (70,), "slots", "", True),
    ("f32", 20, 1, 24, 8, (66, 1), "pages", "", True),
    ("f32", 7, 1, 128, 16, (600, 40), "pages", "counts", False),
    ("f32", 4, 4, 192, 8, (530, 5), "padded", "counts", True),     # fp32 without, several chunks
    ("bf16", 12, 4, 128, 32, (513, 512, 511), "pages", "", True),  # on both sides of one chunk
    ("f16", 4, 2, 32, 1024, (1500, 1), "pages", "", True),         # several chunks to a page
    ("f32", 1, 1, 16, 256, (700,), "slots", "counts", False),
]


def _bias(kind, gen, shape):
    if not kind:
        return None
    x = torch.exp(torch.randn(shape, generator=gen)).ceil().log()
    if kind == "counts":
        x[torch.rand(shape, generator=gen) < 0.3] = -INF
    if kind == "empty":
        x[:] = -INF
    if kind == "lowest":                                   # finite: all alike, an even softmax
        x[:] = torch.finfo(torch.float32).min
        x[0, 0] = 0.0
        x[0, 0, ::2] = torch.finfo(torch.float32).min
    if kind == "huge":
        x[:, :, 5] = 200.0
    return x


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_paged_attention(bench, case):
    dtype, H, K, d, page, lengths, order, bias_kind, want_weights = case
    gen = _gen(H * d + sum(lengths))
    kv, table = C.pool(gen, dtype, K, d, page, lengths, order=order)
    B, cap = len(lengths), max(lengths) + 5
    bias = _bias(bias_kind, gen, (B, K, cap))
    if bias is not None:                                   # what a masked slot holds does not matter
        for b, n in enumerate(lengths):
            for i in range(n):
                for h in range(K):
                    if float(bias[b, h, i]) == -INF:
                        for x in C.cache_views(kv, order, d):
                            x[int(table[b, i // page]), h, i % page] = (math.nan, INF)[i % 2]
            bias[b, :, n:] = math.nan
    q = (torch.randn(B, H, d, generator=gen) * 2).to(TYPES[dtype])
    scale = d ** -0.5
    win = torch.rand(B, K, cap, generator=gen) if want_weights else None
    wout = torch.full((B, K, cap), 9.0) if want_weights else None
    lens = torch.tensor(lengths, dtype=torch.int32)
    want = C.attention_reference(q, *C.cache_views(kv, order, d), table, lens, page, scale, bias, win, wout, dtype)
    got = C.run_attention(bench, q, kv, order, table, lens, scale, bias, win, wout)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")
    if want_weights:
        close(got[2], *want[2], what="weights")
        again = C.run_attention(bench, q, kv, order, table, lens, scale, bias, win, win.clone(), alias=True)   # added up in place
        n = torch.arange(cap) < lens[:, None, None]
        assert torch.equal(torch.where(n, again[2].cpu(), 0.0), torch.where(n, got[2].cpu(), 0.0))
        fresh = C.run_attention(bench, q, kv, order, table, lens, scale, bias, None, wout)
        want0 = C.attention_reference(q, *C.cache_views(kv, order, d), table, lens, page, scale, bias, None, wout, dtype)
        close(fresh[2], *want0[2], what="weights from zero")
        assert torch.equal(fresh[0].cpu(), got[0].cpu())


@pytest.mark.parametrize("dtype,H,K,d", [("bf16", 6, 2, 40), ("f32", 2, 2, 24), ("f32", 9, 3, 64)])
def test_paged_attention_of_rows_with_gaps_and_without_lse(bench, dtype, H, K, d):
    """Queries and results whose rows lie further apart; what is between them stays."""
    gen, lib, page, lengths = _gen(d), bench.lib, 16, (37, 600, 0)
    kv, table = C.pool(gen, dtype, K, d, page, lengths)
    lens, B, gap = torch.tensor(lengths, dtype=torch.int32), len(lengths), 24
    q = torch.randn(B, H * d + gap, generator=gen).to(TYPES[dtype])
    out = bench.guarded(torch.full_like(q, 5.0))
    rows = lambda t: t[:, :H * d].unflatten(1, (H, d))   # noqa: E731
    cache, seqs = lib.PagedCache(*[bench.put(x) for x in kv]), lib.Sequences(bench.put(table), bench.put(lens), max(lengths))
    bench.ctx.sttm_paged_attention(rows(bench.put(q)), cache, seqs, rows(out), 0.2,
                                   workspace=bench.workspace(lib.sttm_paged_attention_workspace_bytes(cache, seqs, H)))
    bench.done()
    want = C.attention_reference(rows(q), *kv, table, lens, page, 0.2, None, None, None, dtype)
    close(rows(out), *want[0], what="out")
    assert (out[:, H * d:] == 5.0).all()


def test_paged_attention_with_pages_outside_of_the_pool(bench):
    """Their slots count as masked, in the middle of a sequence and all over one."""
    gen = _gen(5)
    lengths = (61, 40)
    kv, table = C.pool(gen, "bf16", 2, 64, 8, lengths)
    table[0, 2], table[0, 5], table[0, 7] = -1, kv[0].shape[0], 2 ** 31 - 1
    table[1, :5] = -1
    lens = torch.tensor(lengths, dtype=torch.int32)
    q = torch.randn(2, 4, 64, generator=gen).to(torch.bfloat16)
    win, wout = torch.rand(2, 2, 64, generator=gen), torch.zeros(2, 2, 64)
    want = C.attention_reference(q, *kv, table, lens, 8, 0.125, None, win, wout, "bf16")
    got = C.run_attention(bench, q, kv, "pages", table, lens, 0.125, None, win, wout)
    for name, g, w in zip(("out", "lse", "weights"), got, want):
        close(g, *w, what=name)
    assert (got[0][1] == 0).all() and (got[1][1] == -INF).all()


def test_paged_attention_reads_no_further_than_max_len_and_the_table(bench):
    gen = _gen(6)
    kv, table = C.pool(gen, "f32", 1, 16, 8, (30, 20))
    lens = torch.tensor([30, 10 ** 6], dtype=torch.int32)
    q = torch.randn(2, 2, 16, generator=gen)
    want = C.attention_reference(q, *kv, table[:, :2], lens, 8, 1.0, None, None, None, "f32", max_len=13)
    got = C.run_attention(bench, q, kv, "pages", table[:, :2], lens, 1.0, max_len=13)
    close(got[0], *want[0], what="out")
    want = C.attention_reference(q, *kv, table[:, :2], lens, 8, 1.0, None, None, None, "f32", max_len=16)
    got = C.run_attention(bench, q, kv, "pages", table[:, :2], lens, 1.0)
    close(got[0], *want[0], what="out")
    got = C.run_attention(bench, q, kv, "pages", table, torch.tensor([-3, 0], dtype=torch.int32), 1.0)
    assert (got[0] == 0).all() and (got[1] == -INF).all()


def test_paged_attention_of_values_that_are_not_finite(bench):
    """As the formula has it: an infinite value in a slot that counts, a NaN in a key."""
    gen = _gen(7)
    kv, table = C.pool(gen, "bf16", 2, 32, 8, (40,))
    kv[1][int(table[0, 1]), 0, 3, 5] = INF
    kv[0][int(table[0, 2]), 1, 4, 7] = math.nan
    q = torch.randn(1, 2, 32, generator=gen).to(torch.bfloat16)
    got = C.run_attention(bench, q, kv, "pages", table, torch.tensor([40], dtype=torch.int32), 0.1)
    out = got[0].cpu()
    assert out[0, 0, 5] == INF and torch.isfinite(out[0, 0, :5]).all() and torch.isfinite(out[0, 0, 6:]).all()
    assert torch.isnan(out[0, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,bias_kind", [((1, 40), ""), ((530, 33), ""), ((90, 200), "counts")])
@pytest.mark.parametrize("d", [32, 136])
def test_paged_attention_of_infinite_values(bench, dtype, lengths, bias_kind, d):
    """Every weight is above zero: infinities of one sign give it, whatever the weights' last bits are; both signs or a NaN
    give NaN; what a masked slot holds does not matter; the other channels are as they are."""
    for seed in range(2):
        gen = _gen(100 * d + seed)
        kv, table = C.pool(gen, dtype, 2, d, 8, lengths)
        bias = _bias(bias_kind, gen, (2, 2, max(lengths)))
        if bias is not None:
            bias[:, :, 0] = 0.0
        for b, n in enumerate(lengths):
            for h in range(2):
                slots = [i for i in range(n) if bias is None or float(bias[b, h, i]) != -INF]
                some = [slots[int(x)] for x in torch.randint(0, len(slots), (6,), generator=gen)]
                for i, channel, value in ((some[0], 3, INF), (some[1], 8, -INF), (some[2], 17, INF), (some[3], 17, -INF), (some[4], 30, math.nan),
                                          (some[5], 31, INF)):
                    kv[1][int(table[b, i // 8]), h, i % 8, channel] = value
                for i in range(n):
                    if i not in slots:
                        kv[1][int(table[b, i // 8]), h, i % 8] = (-INF, math.nan)[i % 2]
        q = torch.randn(2, 6, d, generator=gen).to(TYPES[dtype])
        lens = torch.tensor(lengths, dtype=torch.int32)
        want = C.attention_reference(q, *kv, table, lens, 8, 0.1, bias, None, None, dtype)
        got = C.run_attention(bench, q, kv, "pages", table, lens, 0.1, bias)
        close(got[0], *want[0], what=f"out, seed {seed}")
        close(got[1], *want[1], what=f"lse, seed {seed}")


@pytest.mark.parametrize("dtype,q_heads,kv_heads", [("bf16", 4, 2), ("bf16", 17, 1), ("f16", 2, 2), ("f32", 2, 2), ("f32", 6, 2)])
@pytest.mark.parametrize("n", [1, 40, 530])
@pytest.mark.parametrize("bias_kind", ["", "lowest"])
def test_paged_attention_of_scores_that_are_all_nan(bench, dtype, q_heads, kv_heads, n, bias_kind):
    """NaN in the result, the weights and lse alike: -inf stands for no key left, and a part with it would be left out by who
    joins parts. The other sequence is as it is."""
    gen = _gen(n)
    kv, table = C.pool(gen, dtype, kv_heads, 24, 8, (n, 9))
    for i in range(n):
        kv[0][int(table[0, i // 8]), :, i % 8, 2] = math.nan
    bias = _bias(bias_kind, gen, (2, kv_heads, max(n, 9)))
    q, lens = torch.randn(2, q_heads, 24, generator=gen).to(TYPES[dtype]), torch.tensor([n, 9], dtype=torch.int32)
    out, lse, weights = C.run_attention(bench, q, kv, "pages", table, lens, 0.2, bias, None, torch.zeros(2, kv_heads, max(n, 9)))
    want = C.attention_reference(q, *kv, table, lens, 8, 0.2, bias, None, torch.zeros(2, kv_heads, max(n, 9)), dtype)
    for name, g, w in zip(("out", "lse", "weights"), (out, lse, weights), want):
        close(g, *w, what=name)
    assert torch.isnan(lse[0]).all() and torch.isnan(out[0]).all() and torch.isnan(weights[0, :, :n]).all() and torch.isfinite(lse[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [200, 700])
def test_paged_attention_of_many_small_weights(bench, dtype, n):
    """Weights far below the largest one count together: one key of a high score whose value is zero, and slots of 2^-20 to
    2^-34 of its weight with large values, which alone make up the result. Tolerance: a weight's own rounding (scores of up to
    24: 24 * 20 e; two numbers of 16 bits: at least 15 bits together), and the result's."""
    gen = _gen(n)
    kv, table = C.pool(gen, dtype, 1, 16, 8, (n,))
    q = torch.zeros(1, 2, 16)
    q[0, 0, 0], q[0, 1, 0] = 1.0, 0.75
    small = torch.rand(n, generator=gen) * 1.4
    for i in range(n):
        at = int(table[0, i // 8]), 0, i % 8
        kv[0][at], kv[1][at] = 0.0, 30000.0
        kv[0][at][0] = small[i]
    top = n // 3
    kv[0][int(table[0, top // 8]), 0, top % 8, 0] = 24.0
    kv[1][int(table[0, top // 8]), 0, top % 8] = 0.0
    q, lens = q.to(TYPES[dtype]), torch.tensor([n], dtype=torch.int32)
    want = C.attention_reference(q, *kv, table, lens, 8, 1.0, None, None, None, dtype)[0][0]
    got = C.run_attention(bench, q, kv, "pages", table, lens, 1.0)[0]
    assert float(want.min()) > 1e-4      # (above the smallest normal fp16 number)
    close(got, want, want * (24 * 20 * C.E + 2.0 ** -15 + n * C.E + U[dtype] * 1.1) + 2.0 ** -25, what="out")


@pytest.mark.parametrize("dtype,heads", [("bf16", 2), ("f16", 2), ("f32", 1), ("f32", 3)])
@pytest.mark.parametrize("n", [20, 530])
@pytest.mark.parametrize("with_bias", [False, True])
def test_paged_attention_of_scores_near_the_largest_number(bench, dtype, heads, n, with_bias):
    """Scores of 3e38, 0 and -3e38 are finite numbers of 32 bits: the first ones share the weight."""
    gen = _gen(n)
    kv, table = C.pool(gen, dtype, 1, 8, 8, (n,))
    for i in range(n):
        kv[0][int(table[0, i // 8]), 0, i % 8] = 0.0
        kv[0][int(table[0, i // 8]), 0, i % 8, 0] = (0.0, 1.0, -1.0)[i % 3]
    q = torch.zeros(1, heads, 8)
    q[:, :, 0] = 1.0
    q, lens, bias = q.to(TYPES[dtype]), torch.tensor([n], dtype=torch.int32), torch.zeros(1, 1, n) if with_bias else None
    zero = torch.zeros(1, 1, n)
    want = C.attention_reference(q, *kv, table, lens, 8, 3e38, bias, None, zero, dtype)
    got = C.run_attention(bench, q, kv, "pages", table, lens, 3e38, bias, None, zero)
    some = torch.arange(n) % 3 == 1
    even = torch.stack([kv[1][int(table[0, i // 8]), 0, i % 8] for i in range(n) if i % 3 == 1]).double().mean(0)
    assert torch.allclose(want[0][0][0, 0], even)
    for name, g, w in zip(("out", "lse", "weights"), got, want):
        close(g, w[0], {"out": 2 * U[dtype] * 4.0, "lse": 1e32, "weights": 1e-5}[name], what=name)
    assert (got[2].cpu()[0, 0][~some] == 0).all()


# -- eviction ----------------------------------------------------------------------------------------------------------

EVICT = [
    # dtype, kv_heads, d, page, lengths, keep, sink, recent, ids, bias, weights, order
    ("bf16", 2, 128, 16, (40, 1, 0), (20, 1, 0), 4, 8, "none", False, "spread", "pages"),
    ("f32", 3, 72, 8, (100, 33), (99, 0), 0, 0, "again", True, "spread", "slots"),       # one goes; all go
    ("f16", 1, 80, 8, (64, 65), (70, 64), 2, 5, "again", True, "ties", "padded"),        # none goes; ties
    ("bf16", 1, 8, 8, (1100,), (500,), 16, 100, "minus", False, "ties", "pages"),        # several rounds of a workgroup
    ("f32", 1, 256, 32, (50,), (30,), 20, 25, "minus", True, "spread", "pages"),         # more protected than stay
    ("bf16", 2, 64, 64, (90, 70), (45, 1), 0, 1, "again", False, "odd", "slots"),        # NaN, infinities, both zeros
    ("f16", 2, 40, 8, (30,), (-4,), 0, 0, "none", True, "spread", "pages"),
    ("bf16", 1, 16, 8, (77,), (33,), 0, 0, "again", False, "equal", "pages"),
    ("bf16", 2, 8, 64, (4097,), (4096,), 4, 64, "again", False, "zeros", "pages"),       # one goes, of many that are alike
    ("f32", 1, 8, 64, (9001, 8193), (4500, 8192), 4, 64, "again", True, "zeros", "pages"),   # rows of several workgroups
    ("bf16", 1, 8, 64, (8200, 33), (100, 5), 0, 0, "minus", False, "equal", "pages"),
    ("bf16", 1, 8, 64, (6000,), (2500,), 3, 40, "again", False, "equal", "pages"),       # more alike than the list holds
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
@pytest.mark.parametrize("alias", [False, True])
def test_cache_evict(bench, case, alias):
    dtype, K, d, page, lengths, keep, sink, recent, ids_kind, with_bias, w_kind, order = case
    gen = _gen(sum(lengths) + d)
    kv, table = C.pool(gen, dtype, K, d, page, lengths, order=order, junk=3.0)
    B, cap = len(lengths), max(lengths) + 3
    w = torch.randn(B, K, cap, generator=gen).exp()
    if w_kind == "ties":
        w = torch.randint(0, 3, (B, K, cap), generator=gen).float()
    if w_kind == "equal":
        w = torch.full((B, K, cap), 0.25)
    if w_kind == "zeros":
        w = torch.where(torch.rand(B, K, cap, generator=gen) < 0.1, 0.0, w)
    if w_kind == "odd":
        some = torch.tensor([math.nan, -math.nan, INF, -INF, 0.0, -0.0, 1e-42, -1.0])
        w = some[torch.randint(0, 8, (B, K, cap), generator=gen)]
    total = torch.tensor([n + 50 for n in lengths], dtype=torch.int32) if ids_kind != "none" else None
    ids = None if ids_kind == "none" else torch.full((B, K, cap), -1, dtype=torch.int32)
    if ids_kind == "again":
        for b, n in enumerate(lengths):
            for h in range(K):
                ids[b, h, :n // 2] = torch.randperm(50 + n // 2, generator=gen)[:n // 2].to(torch.int32)
    if alias and ids is None:
        ids = torch.full((B, K, cap), -1, dtype=torch.int32)
    bias = torch.randn(B, K, cap, generator=gen) if with_bias else None
    lens, keeps = torch.tensor(lengths, dtype=torch.int32), torch.tensor(keep, dtype=torch.int32)
    outs = [w, ids, bias] if alias else [torch.full_like(w, 5.0), torch.full((B, K, cap), 5, dtype=torch.int32), None if bias is None else torch.full_like(w, 5.0)]
    want = C.evict_reference(*C.cache_views(kv, order, d), table, lens, page, keeps, total, sink, recent, w, ids, bias, *outs)
    got = C.run_evict(bench, kv, order, d, table, lens, keeps, total, sink, recent, w, ids, bias, *outs, alias=alias)
    for name, g, x in zip(("k", "v", "weights", "ids", "bias", "lengths"), got, want):
        if x is not None:
            g = g.cpu()
            same = (g == x) | (torch.isnan(g) & torch.isnan(x)) if g.is_floating_point() else g == x
            assert same.all(), name


def test_cache_evict_of_numbers_that_occur_twice(bench):
    """Not allowed: which of them stay is open, but the lengths are as they have to be and nothing else is touched."""
    gen = _gen(13)
    n, keep = 300, 120
    kv, table = C.pool(gen, "bf16", 1, 8, 8, (n,), junk=3.0)
    w, ids = torch.zeros(1, 1, n), torch.full((1, 1, n), 7, dtype=torch.int32)
    lens = torch.tensor([n], dtype=torch.int32)
    outs = [torch.zeros_like(w), torch.zeros_like(ids), None]
    got = C.run_evict(bench, kv, "pages", 8, table, lens, torch.tensor([keep], dtype=torch.int32), None, 0, 0, w, ids, None, *outs)
    assert got[5].tolist() == [keep] and (got[3][0, 0, :keep] == 7).sum() <= keep


@pytest.mark.parametrize("n,keep", [(60, 31), (300, 121), (1100, 1099), (5000, 2501), (9001, 101), (9001, 8999)])
@pytest.mark.parametrize("times,w_kind", [(2, "equal"), (5, "equal"), (3, "ties")])
def test_cache_evict_leaves_whole_tables_where_numbers_occur_twice(bench, n, keep, times, w_kind):
    """Which of the slots of one number stay is open. Everything else is as ever: the other numbers that stay, every token with
    its own row and weight, no slot twice, and nothing left behind the new length."""
    gen = _gen(n + times)
    kv, table = C.pool(gen, "f32", 1, 8, 64, (n,), junk=-5.0)
    perm = torch.randperm(n, generator=gen)
    ids = torch.zeros(1, 1, n, dtype=torch.int32)
    ids[0, 0, perm] = (torch.arange(n) // times).to(torch.int32)
    w = torch.full((1, 1, n), 0.5) if w_kind == "equal" else (ids % 3).float()     # (alike where the numbers are)
    for i in range(n):
        kv[0][int(table[0, i // 64]), 0, i % 64], kv[1][int(table[0, i // 64]), 0, i % 64] = float(i), -float(i)
    lens, keeps = torch.tensor([n], dtype=torch.int32), torch.tensor([keep], dtype=torch.int32)
    outs = [torch.full_like(w, 9.0), torch.full_like(ids, 9), None]
    k, v, w2, ids2, _, new = [x if x is None else x.cpu() for x in
                              C.run_evict(bench, kv, "pages", 8, table, lens, keeps, None, 0, 0, w, ids, None, *outs)]
    assert new.tolist() == [keep]
    want = sorted(range(n), key=lambda i: (-float(w[0, 0, i]), int(ids[0, 0, i])))[:keep]
    assert sorted(ids2[0, 0, :keep].tolist()) == sorted(ids[0, 0, want].tolist())
    fro = torch.stack([k[int(table[0, i // 64]), 0, i % 64, 0] for i in range(keep)]).long()
    assert len(set(fro.tolist())) == keep and torch.equal(ids[0, 0, fro], ids2[0, 0, :keep]) and torch.equal(w[0, 0, fro], w2[0, 0, :keep])
    assert torch.equal(torch.stack([v[int(table[0, i // 64]), 0, i % 64, 0] for i in range(keep)]).long(), -fro)
    assert (ids2[0, 0, keep:] == -1).all() and (w2[0, 0, keep:] == 0).all()


def test_cache_evict_among_protected_slots_goes_by_their_numbers(bench):
    """Fewer stay than are protected: the lowest numbers do, whatever the weights."""
    gen, n = _gen(15), 100
    kv, table = C.pool(gen, "f32", 1, 8, 8, (n,), junk=3.0)
    w = torch.arange(n).float()[None, None].clone()
    lens, keep = torch.tensor([n], dtype=torch.int32), torch.tensor([12], dtype=torch.int32)
    ids = C.run_evict(bench, kv, "pages", 8, table, lens, keep, None, 4, 32, w, None, None, torch.zeros_like(w), torch.zeros(1, 1, n, dtype=torch.int32),
                      None)[3].cpu()
    assert sorted(ids[0, 0, :12].tolist()) == [0, 1, 2, 3, 68, 69, 70, 71, 72, 73, 74, 75]


def test_cache_evict_with_pages_outside_of_the_pool(bench):
    """Their slots take part in the order; rows are neither read from nor written to them."""
    gen = _gen(11)
    kv, table = C.pool(gen, "f32", 1, 8, 8, (48,), junk=3.0)
    table[0, 0], table[0, 4] = -2, kv[0].shape[0] + 5
    w = torch.rand(1, 1, 48, generator=gen)
    lens, keep = torch.tensor([48], dtype=torch.int32), torch.tensor([20], dtype=torch.int32)
    outs = [torch.zeros_like(w), torch.zeros(1, 1, 48, dtype=torch.int32), None]
    want = C.evict_reference(*kv, table, lens, 8, keep, None, 0, 0, w, None, None, *outs)
    got = C.run_evict(bench, kv, "pages", 8, table, lens, keep, None, 0, 0, w, None, None, *outs)
    for g, x in zip(got, want):
        assert x is None or torch.equal(g.cpu(), x)


def test_cache_evict_without_slots(bench):
    """No pages, or no length at all: the lengths are zero, the tables are as they were."""
    gen = _gen(14)
    kv, table = C.pool(gen, "bf16", 2, 8, 8, (9,), junk=3.0)
    w, keep, lens = torch.rand(1, 2, 9, generator=gen), torch.tensor([4], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    for t in (table, table[:, :0].clone()):
        outs = [torch.full_like(w, 5.0), torch.full((1, 2, 9), 5, dtype=torch.int32), None]
        got = C.run_evict(bench, kv, "pages", 8, t, lens, keep, None, 0, 0, w, None, None, *outs)
        for g, x in zip(got, (*kv, outs[0], outs[1], None, lens)):
            assert x is None or torch.equal(g.cpu(), x)


def test_eviction_then_attention_over_what_stays(bench):
    """The slots that stay, in whatever order, give what attention over those tokens alone gives."""
    gen = _gen(12)
    n, keep, page, d = 83, 41, 8, 32
    kv, table = C.pool(gen, "f32", 2, d, page, (n,), junk=0.0)
    q = torch.randn(1, 4, d, generator=gen)
    lens = torch.tensor([n], dtype=torch.int32)
    zero = torch.zeros(1, 2, n)
    w = C.run_attention(bench, q, kv, "pages", table, lens, 0.3, None, None, zero)[2].cpu()
    ids = torch.zeros(1, 2, n, dtype=torch.int32)
    k, v, w2, ids2, _, new = C.run_evict(bench, kv, "pages", d, table, lens, torch.tensor([keep], dtype=torch.int32), None, 1, 2, w, None, None,
                                         zero, ids, None)
    assert new.tolist() == [keep]
    out, lse, _ = C.run_attention(bench, q, [k.cpu(), v.cpu()], "pages", table, new.cpu(), 0.3)
    mask = torch.full((1, 2, n), -INF)
    for h in range(2):
        kept = ids2[0, h, :keep].cpu().tolist()
        assert len(set(kept)) == keep and {0, n - 2, n - 1} <= set(kept)
        mask[0, h, kept] = 0.0
    want = C.attention_reference(q, *kv, table, lens, page, 0.3, mask, None, None, "f32")
    close(out, *want[0], what="out")
    close(lse, *want[1], what="lse")


# -- refusals ----------------------------------------------------------------------------------------------------------

def _refused(bench, code, call, *args, **kw):
    with pytest.raises(bench.lib.SttmError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_refusals_of_descriptions(bench):
    lib = bench.lib
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    _refused(bench, lib.STTM_ERR_SHAPE, lib.PagedCache, z(2, 1, 8, 16), z(2, 1, 8, 24))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.PagedCache, z(2, 1, 16, 8).transpose(2, 3), z(2, 1, 16, 8).transpose(2, 3))
    _refused(bench, lib.STTM_ERR_DTYPE, lib.PagedCache, z(2, 1, 8, 16), z(2, 1, 8, 16, dtype=torch.float16))
    _refused(bench, lib.STTM_ERR_DTYPE, lib.PagedCache, z(2, 1, 8, 16, dtype=torch.int32), z(2, 1, 8, 16, dtype=torch.int32))
    _refused(bench, lib.STTM_ERR_DTYPE, lib.Sequences, z(2, 4), z(2, dtype=torch.int32))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.Sequences, z(2, 4, dtype=torch.int32), z(3, dtype=torch.int32))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.Sequences, z(2, 4, dtype=torch.int32), z(2, dtype=torch.int32), -1)
    _refused(bench, lib.STTM_ERR_DTYPE, lib.Rope, z(3, dtype=torch.int64), z(4))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.Rope, z(3, 1), z(4), (2, 2))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.Rope, z(3, 3), z(4), (2, 3))


def test_refusals_of_the_library(bench):
    """What the C entries themselves refuse, with their codes; nothing is launched."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    seqs = lib.Sequences(z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32))
    for shape in ((2, 1, 8, 12), (2, 1, 8, 264), (2, 1, 4, 16), (2, 1, 24, 16), (2, 1, 2048, 8), (2, 1025, 8, 8)):
        cache = lib.PagedCache(z(*shape), z(*shape))
        assert lib.sttm_paged_attention_workspace_bytes(cache, seqs, shape[1]) == 0 and lib.sttm_cache_evict_workspace_bytes(cache, seqs) == 0
        _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, z(1, shape[1], shape[3]), cache, seqs, z(1, shape[1], shape[3]), 1.0)
    odd = z(2 * 8 * 16 + 1)[1:].view(2, 1, 8, 16)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_paged_attention, z(1, 1, 16), lib.PagedCache(odd, odd), seqs, z(1, 1, 16), 1.0)
    wide = z(2, 1, 8, 18)[..., :16]
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, z(1, 1, 16), lib.PagedCache(wide, wide), seqs, z(1, 1, 16), 1.0)

    far = lib.PagedCache(z(1, 1, 1024, 16), z(1, 1, 1024, 16))
    far.struct.token_stride = 1 << 20                              # (described only: refused before anything is read)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, z(1, 1, 16), far, seqs, z(1, 1, 16), 1.0)

    cache = lib.PagedCache(z(2, 2, 8, 16), z(2, 2, 8, 16))
    ws = bench.workspace(1 << 16)
    ok = dict(workspace=ws)
    q = z(1, 4, 16)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), 1.0)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), 1.0, workspace=ws[:128])
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), 1.0, workspace=ws[1:])
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, z(1, 3, 16), cache, seqs, z(1, 3, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), 1.0, key_bias=z(1, 2, 15), **ok)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), math.nan, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 24), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, ctx.sttm_paged_attention, q.half(), cache, seqs, z(1, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, q, cache, seqs, z(1, 4, 16), 1.0, weights_out=z(1, 1, 16), **ok)

    i = lambda *s: z(*s, dtype=torch.int32)   # noqa: E731
    t, n = z(1, 2, 16), i(1, 2, 16)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_cache_evict, cache, seqs, i(1), i(1), t, t, n, n, sink=-1, **ok)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_cache_evict, cache, seqs, i(1), i(1), t, t, n, n, bias_in=t, **ok)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_cache_evict, cache, seqs, i(1), i(1), t, t, n, n)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cache_evict, cache, seqs, i(2), i(1), t, t, n, n, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cache_evict, cache, seqs, i(1), i(1), z(1, 2, 9), z(1, 2, 9), i(1, 2, 9), i(1, 2, 9), **ok)

    k = z(3, 2, 16)
    slots = z(3, dtype=torch.int64)
    rope = lib.Rope(i(3), z(8))
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_qk_norm_rope, z(3, 4, 16), k, k, z(3, 4, 16), eps=-1.0)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_qk_norm_rope, z(3, 4, 16), k, k, z(3, 4, 16), cache=cache)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 16), k, k, z(3, 4, 16), rope=lib.Rope(i(3), z(12)))
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 16), k, k, z(3, 4, 16), rope=lib.Rope(i(3), z(6)))
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 16), k, k, z(3, 4, 16), rope=lib.Rope(i(2), z(8)))
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 12), z(3, 2, 12), k, z(3, 4, 12))
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 16), z(3, 1, 16), z(3, 1, 16), z(3, 4, 16), cache=cache, slots=slots, rope=rope)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_qk_norm_rope, z(3, 4, 16).transpose(0, 1), k, k, z(3, 4, 16))
    _refused(bench, lib.STTM_ERR_DTYPE, ctx.sttm_qk_norm_rope, z(3, 4, 16), k.half(), k, z(3, 4, 16))
    bench.done()


def test_nothing_to_do(bench):
    """No rows, no sequences: no launch, no error."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    cache = lib.PagedCache(z(2, 2, 8, 16), z(2, 2, 8, 16))
    seqs = lib.Sequences(z(0, 2, dtype=torch.int32), z(0, dtype=torch.int32))
    ctx.sttm_qk_norm_rope(z(0, 4, 16), z(0, 2, 16), z(0, 2, 16), z(0, 4, 16), cache=cache, slots=z(0, dtype=torch.int64))
    ctx.sttm_paged_attention(z(0, 4, 16), cache, seqs, z(0, 4, 16), 1.0)
    n = z(0, dtype=torch.int32)
    ctx.sttm_cache_evict(cache, seqs, n, n, z(0, 2, 16), z(0, 2, 16), None, z(0, 2, 16, dtype=torch.int32))


def test_large_batches_without_a_max_len(bench):
    """Without max_len a sequence ends with its row of the table, and that is what counts in the limits of a call."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    batch, H, K = 1500, 64, 8
    cache = lib.PagedCache(z(2, K, 8, 8), z(2, K, 8, 8))
    table = torch.ones(batch, 1, dtype=torch.int32)
    seqs = lib.Sequences(bench.put(table), z(batch, dtype=torch.int32))
    assert lib.sttm_paged_attention_workspace_bytes(cache, seqs, H, True) > 0 and lib.sttm_cache_evict_workspace_bytes(cache, seqs) > 0
    w, ids, n = z(batch, K, 8), z(batch, K, 8, dtype=torch.int32), z(batch, dtype=torch.int32)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_paged_attention, z(batch, H, 8), cache, seqs, z(batch, H, 8), 1.0)   # (the last thing asked for)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_cache_evict, cache, seqs, n, n, w, w, ids, ids)


def test_refusals_of_what_is_too_large(bench):
    """Described only: refused before anything is read."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    cache, q = lib.PagedCache(z(2, 8, 8, 8), z(2, 8, 8, 8)), z(1, 64, 8)
    seqs = lib.Sequences(z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32))
    seqs.struct.batch, seqs.struct.max_pages, seqs.struct.table_stride = 60000, 1 << 26, 1 << 26
    assert lib.sttm_paged_attention_workspace_bytes(cache, seqs, 64, True) == 0 and lib.sttm_cache_evict_workspace_bytes(cache, seqs) == 0
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, q, cache, seqs, q, 1.0)


def test_refusals_of_sequences_that_slot_numbers_do_not_reach(bench):
    """Slots are numbered in 32 bits, twice as many as a sequence may have: 2^30 are the most. Described only."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    cache, q = lib.PagedCache(z(2, 1, 8, 8), z(2, 1, 8, 8)), z(1, 1, 8)
    seqs = lib.Sequences(z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32))
    t, i = z(1, 1, 16), z(1, 1, 16, dtype=torch.int32)
    n = z(1, dtype=torch.int32)
    for pages, max_len, ok in ((1 << 27, 2 ** 31 - 1, True), ((1 << 27) + 1, 2 ** 31 - 1, False), ((1 << 28) - 1, 1 << 30, True),
                               ((1 << 28) - 1, (1 << 30) + 1, False), (2, 2 ** 31 - 1, True)):
        seqs.struct.max_pages, seqs.struct.table_stride, seqs.struct.max_len = pages, pages, max_len
        sizes = [lib.sttm_paged_attention_workspace_bytes(cache, seqs, 1, True), lib.sttm_cache_evict_workspace_bytes(cache, seqs)]
        assert (min(sizes) > 0) == ok and (max(sizes) > 0) == ok
        if not ok:
            _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_paged_attention, q, cache, seqs, q, 1.0)
            _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cache_evict, cache, seqs, n, n, t, t, i, i)
