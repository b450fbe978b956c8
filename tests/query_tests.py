"""Tests of the attention of several queries that run on the GPU (test_queries_gpu.py) and on host threads
(test_queries_cpu.py): `bench` is the context under test."""
import math

import pytest
import torch

from tests import cache_cases as C
from tests import query_cases as Q
from tests.cache_cases import INF, TYPES, close


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bias(kind, gen, shape):
    x = torch.exp(torch.randn(shape, generator=gen)).ceil().log()
    if kind == "counts":
        x[torch.rand(shape, generator=gen) < 0.3] = -INF
    if kind == "empty":
        x[:] = -INF
    if kind == "lowest":                                   # finite: all alike, an even softmax
        x[:] = torch.finfo(torch.float32).min
    if kind == "huge":
        x[..., 3::7] = 200.0
    return x


# -- packed states -----------------------------------------------------------------------------------------------------

CROSS = [
    # dtype, q_heads, kv_heads, d, tokens (None: one each), states, layout, bias, bias by head
    ("bf16", 7, 1, 128, None, (1,), "projection", "", False),
    ("bf16", 14, 2, 128, None, (33, 0, 300), "projection", "counts", False),
    ("f16", 4, 2, 80, (3, 1, 0, 2), (31, 32, 5, 129), "heads", "", False),
    ("f32", 3, 3, 72, (5, 2), (5, 160), "projection", "counts", True),
    ("f32", 2, 1, 256, (1, 40), (17, 70), "gap", "", False),
    ("bf16", 2, 2, 256, (9, 33), (65, 40), "projection", "counts", True),
    ("f16", 1, 1, 8, None, (1, 257), "projection", "counts", False),
    ("bf16", 17, 1, 64, (2, 13), (70, 3), "heads", "counts", False),
    ("f16", 33, 1, 40, (5,), (200,), "gap", "huge", True),
    ("f32", 5, 5, 24, (2, 3), (0, 0), "projection", "", False),      # no states at all
    ("bf16", 8, 4, 96, (65, 4), (64, 129), "projection", "lowest", False),
    ("f32", 4, 2, 136, (7,), (67,), "heads", "empty", False),
    ("f16", 3, 1, 168, (44,), (45,), "projection", "empty", True),
    ("bf16", 2, 1, 192, (70,), (100,), "projection", "", False),
    ("f32", 6, 2, 192, (12, 1), (90, 33), "projection", "", False),
    ("f32", 1, 1, 128, (130,), (66,), "gap", "counts", True),
    ("f16", 2, 2, 32, (260,), (64,), "projection", "", False),        # several tiles of rows
    ("bf16", 5, 1, 136, (1, 1, 1), (40, 0, 7), "projection", "counts", False),
]


@pytest.mark.parametrize("case", CROSS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_cross_attention(bench, case):
    dtype, H, K, d, tokens, lengths, layout, bias_kind, by_head = case
    gen = _gen(H * d + sum(lengths))
    rows, gap = sum(lengths) + 9, 0 if tokens is None else 2             # (rows behind the last sequence, tokens around them)
    storage, view = Q.states(gen, dtype, K, d, rows, layout)
    offsets = Q.offsets_of(lengths, 4)
    q_offsets = None if tokens is None else Q.offsets_of(tokens, gap)
    T = len(lengths) if tokens is None else sum(tokens) + 2 * gap
    q = (torch.randn(T, H, d, generator=gen) * 2).to(TYPES[dtype])
    bias = _bias(bias_kind, gen, (K, rows) if by_head else (rows,)) if bias_kind else None
    k, v = view(storage)
    if bias is not None:                                   # what a masked state holds does not matter
        masked = bias == -INF if by_head else (bias == -INF).expand(K, rows)
        for h in range(K):
            for i in masked[h].nonzero().flatten().tolist():
                k[i, h], v[i, h] = (math.nan, INF)[i % 2], (INF, math.nan)[i % 2]
        bias[..., sum(lengths) + 4:] = math.nan
    for x in (k, v):                                       # nor what stands around the sequences
        x[:4], x[sum(lengths) + 4:] = math.nan, INF
    scale = d ** -0.5
    seven = torch.full((T, H, d), 7.0), torch.full((T, H), 7.0)
    want = Q.cross_reference(q, q_offsets, k, v, offsets, scale, bias, *seven, dtype)
    got = Q.run_cross(bench, q, q_offsets, storage, view, offsets, scale, bias)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


def test_cross_attention_reads_no_further_than_max_rows_and_the_buffers(bench):
    gen = _gen(2)
    storage, view = Q.states(gen, "f32", 1, 16, 50, "projection")
    q = torch.randn(2, 2, 16, generator=gen)
    seven = torch.full((2, 2, 16), 7.0), torch.full((2, 2), 7.0)
    want = Q.cross_reference(q, None, *view(storage), torch.tensor([0, 30, 50]), 1.0, None, *seven, "f32", max_rows=13)
    got = Q.run_cross(bench, q, None, storage, view, torch.tensor([0, 30, 50]), 1.0, max_rows=13)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")
    want = Q.cross_reference(q, None, *view(storage), torch.tensor([0, 30, 50]), 1.0, None, *seven, "f32")
    got = Q.run_cross(bench, q, None, storage, view, torch.tensor([-5, 30, 10 ** 12]), 1.0)
    close(got[0], *want[0], what="out")
    # tokens behind the last row are not there either, nor are states that end before they begin
    got = Q.run_cross(bench, q, torch.tensor([1, 2, 900]), storage, view, torch.tensor([40, 20, 30]), 1.0)
    assert (got[0][1] == 0).all() and (got[1][1] == -INF).all() and (got[0][0] == 7).all() and (got[1][0] == 7).all()


@pytest.mark.parametrize("dtype,d,tokens", [("bf16", 64, 1), ("f16", 136, 5), ("f32", 72, 40), ("bf16", 40, 130)])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-35, 3e-4])
def test_cross_attention_at_any_scale(bench, dtype, d, tokens, scale):
    """No scale at all (every state counts the same), a negative one, one that takes scores below the smallest normal number."""
    gen = _gen(d)
    storage, view = Q.states(gen, dtype, 1, d, 77, "projection")
    q = torch.randn(tokens, 2, d, generator=gen).to(TYPES[dtype])
    seven = torch.full((tokens, 2, d), 7.0), torch.full((tokens, 2), 7.0)
    offsets, q_offsets = Q.offsets_of((77,)), Q.offsets_of((tokens,))
    want = Q.cross_reference(q, q_offsets, *view(storage), offsets, scale, None, *seven, dtype)
    got = Q.run_cross(bench, q, q_offsets, storage, view, offsets, scale)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


@pytest.mark.parametrize("dtype,heads,tokens", [("bf16", 2, 1), ("f16", 2, 70), ("f32", 1, 3), ("f32", 3, 50)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("big", [3e38, 3e30])
def test_cross_attention_of_scores_near_the_largest_number(bench, dtype, heads, tokens, with_bias, big):
    """Scores of 3e38, 0 and -3e38 are finite numbers of 32 bits: the first ones share the weight. (3e30 as a scale of 1e30 and
    products of 3, or of 3e8 and 1e22.)"""
    n = 100
    storage, view = Q.states(_gen(n), dtype, 1, 8, n, "projection")
    k, v = view(storage)
    k[:] = 0.0
    k[1::3, :, 0], k[2::3, :, 0] = 1.0, -1.0
    q = torch.zeros(tokens, heads, 8)
    q[:, :, 0] = 1.0 if big == 3e38 else 3.0
    scale = 3e38 if big == 3e38 else 1e30
    q, offsets, q_offsets = q.to(TYPES[dtype]), Q.offsets_of((n,)), Q.offsets_of((tokens,))
    got = Q.run_cross(bench, q, q_offsets, storage, view, offsets, scale, torch.zeros(n) if with_bias else None)
    even = v[1::3, 0].double().mean(0).expand(tokens, heads, 8)
    close(got[0], even, 2 * C.U[dtype] * 4.0, what="out")
    close(got[1], torch.full((tokens, heads), big, dtype=torch.float64), 2.0 ** -22 * big, what="lse")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("apart", [1, 2, 4])
def test_cross_attention_of_large_scores_that_rise_by_a_step(bench, dtype, tokens, apart):
    """Scores of 2^23 and 2^23 + 1 (2^24 and 2^24 + 2, 2^25 and + 4): next to each other in 32 bits, the higher ones last."""
    n = 400
    storage, view = Q.states(_gen(n), dtype, 1, 8, n, "projection")
    k, v = view(storage)
    k[:], v[:, :, 0] = 0.0, 1.0
    k[:, :, 0], k[300:, :, 1] = 4096.0, apart
    q = torch.zeros(tokens, 2, 8)
    q[:, :, 0], q[:, :, 1] = 2048.0 * apart, 1.0
    got = Q.run_cross(bench, q.to(TYPES[dtype]), Q.offsets_of((tokens,)), storage, view, Q.offsets_of((n,)), 1.0)
    # all products and sums up to here are exact: an even number of weights of 1 and of e^apart
    w = torch.ones(n, dtype=torch.float64)
    w[300:] = math.exp(apart)
    w = w / w.sum()
    want, size = w @ v[:, 0].double(), w @ v[:, 0].double().abs()
    tol = size * ((n + 64) * C.E + (0 if dtype == "f32" else C.U[dtype])) + C.U[dtype] * 1.02 * want.abs() + (2.0 ** -40 * n * 8 if dtype == "f16" else 0)
    close(got[0], want.expand(tokens, 2, 8), tol.expand(tokens, 2, 8), what="out")


def test_cross_attention_of_large_products(bench):
    """Products of 3e38 at a scale of one, fp32."""
    n, tokens = 70, 4
    storage, view = Q.states(_gen(n), "f32", 1, 8, n, "projection")
    k, v = view(storage)
    k[:] = 0.0
    k[1::3, :, 0], k[2::3, :, 0] = 3e19, -3e19
    q = torch.zeros(tokens, 1, 8)
    q[:, :, 0] = 1e19
    got = Q.run_cross(bench, q, Q.offsets_of((tokens,)), storage, view, Q.offsets_of((n,)), 1.0)
    close(got[0], v[1::3, 0].double().mean(0).expand(tokens, 1, 8), 1e-5, what="out")
    close(got[1], torch.full((tokens, 1), 3e38, dtype=torch.float64), 1e32, what="lse")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens", [1, 45])
@pytest.mark.parametrize("bias_kind", ["", "counts"])
def test_cross_attention_of_values_that_are_not_finite(bench, dtype, tokens, bias_kind):
    """Infinities of one sign give it, both signs or a NaN give NaN, in their channel alone; a NaN in a key makes its head NaN, lse too."""
    gen, n, d = _gen(tokens), 150, 40
    storage, view = Q.states(gen, dtype, 2, d, n, "projection")
    k, v = view(storage)
    bias = _bias(bias_kind, gen, (n,)) if bias_kind else None
    there = [i for i in range(n) if bias is None or float(bias[i]) != -INF]
    for i, channel, value in ((there[3], 3, INF), (there[40], 8, -INF), (there[41], 17, INF), (there[70], 17, -INF), (there[-1], 30, math.nan)):
        v[i, 0, channel] = value
    for i in range(n):
        if i not in there:
            v[i], k[i] = (-INF, math.nan)[i % 2], math.nan
    k[there[5], 1, 7] = math.nan
    q = torch.randn(tokens, 4, d, generator=gen).to(TYPES[dtype])
    seven = torch.full((tokens, 4, d), 7.0), torch.full((tokens, 4), 7.0)
    want = Q.cross_reference(q, Q.offsets_of((tokens,)), k, v, Q.offsets_of((n,)), 0.1, bias, *seven, dtype)
    got = Q.run_cross(bench, q, Q.offsets_of((tokens,)), storage, view, Q.offsets_of((n,)), 0.1, bias)
    assert torch.isnan(want[0][0][:, 2:]).all() and torch.isinf(want[0][0][:, :2, 3]).all() and torch.isnan(want[0][0][:, :2, 17]).all()
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens", [1, 40])
def test_cross_attention_of_many_small_weights(bench, dtype, tokens):
    """One state of a high score whose value is zero, and states of 2^-20 to 2^-33 of its weight with large values, which alone make up the
    result."""
    gen, n = _gen(5), 200
    storage, view = Q.states(gen, dtype, 1, 16, n, "projection")
    k, v = view(storage)
    k[:], v[:] = 0.0, 30000.0
    k[:, 0, 0] = torch.rand(n, generator=gen) * 1.4
    k[n // 3, 0, 0], v[n // 3] = 24.0, 0.0
    q = torch.zeros(tokens, 2, 16)
    q[:, 0, 0], q[:, 1, 0] = 1.0, 0.75
    q = q.to(TYPES[dtype])
    seven = torch.full((tokens, 2, 16), 7.0), torch.full((tokens, 2), 7.0)
    (want, tol), _ = Q.cross_reference(q, Q.offsets_of((tokens,)), k, v, Q.offsets_of((n,)), 1.0, None, *seven, dtype)
    got = Q.run_cross(bench, q, Q.offsets_of((tokens,)), storage, view, Q.offsets_of((n,)), 1.0)[0]
    assert float(want.min()) > 1e-4
    close(got, want, tol + want * 24 * 20 * C.E, what="out")


# -- a shared prefix ---------------------------------------------------------------------------------------------------

SHARED = [
    # dtype, q_heads, kv_heads, d, page, prefix lengths, sequences before each group, own lengths, tokens (None: one each), order, biases
    ("bf16", 7, 1, 128, 16, (40,), (0, 2), (5, 1), None, "pages", ("", "")),
    ("bf16", 14, 2, 128, 16, (130, 0, 33), (0, 2, 3, 5), (3, 70, 1, 9, 200), None, "pages", ("counts", "")),
    ("f16", 4, 2, 80, 8, (31,), (1, 3), (8, 9, 30, 7), (3, 2, 5, 1), "slots", ("", "")),       # sequences of no group
    ("f32", 3, 3, 72, 16, (65, 20), (0, 1, 3), (12, 40, 3), (12, 7, 3), "pages", ("counts", "counts")),
    ("f32", 2, 1, 256, 32, (50,), (0, 2), (34, 36), (2, 36), "padded", ("", "")),
    ("bf16", 2, 2, 256, 8, (33,), (0, 3), (9, 0, 20), (1, 0, 20), "pages", ("", "counts")),
    ("f16", 1, 1, 8, 8, (), (0,), (100, 33), (100, 2), "pages", ("", "")),                      # groups there are none
    ("bf16", 3, 1, 64, 64, None, None, (130, 65), (130, 60), "pages", ("", "")),                # no prefixes: causal alone
    ("f16", 2, 2, 32, 1024, (140,), (0, 2), (200, 66), (129, 66), "slots", ("", "")),
    ("f32", 5, 5, 24, 8, (0,), (0, 2), (0, 3), (1, 5), "pages", ("", "")),                      # more tokens than slots; nothing to see
    ("bf16", 8, 4, 96, 8, (17, 5), (0, 4, 4), (1, 2, 3, 4), None, "pages", ("lowest", "lowest")),
    ("f32", 4, 2, 136, 8, (67,), (0, 2), (5, 4), (5, 4), "slots", ("empty", "")),
    ("bf16", 2, 1, 192, 16, (90,), (0, 2), (40, 70), (40, 33), "pages", ("huge", "")),
    ("f32", 1, 1, 16, 256, (300,), (0, 1), (150,), (140,), "pages", ("", "")),
]


def _shared_case(case, gen):
    dtype, H, K, d, page, lengths, groups, own, tokens, order, biases = case
    all_lengths = (lengths or ()) + own
    kv, table = C.pool(gen, dtype, K, d, page, all_lengths, order=order)
    n = len(lengths or ())
    pre = None if lengths is None else (table[:n].contiguous(), torch.tensor(lengths, dtype=torch.int32))
    mine = (table[n:].contiguous(), torch.tensor(own, dtype=torch.int32))
    views, out = C.cache_views(kv, order, d), []
    for kind, of in ((biases[0], pre), (biases[1], mine)):
        if not kind:
            out.append(None)
            continue
        bias = _bias(kind, gen, (len(of[1]), K, max([1] + of[1].tolist())))
        for b, m in enumerate(of[1].tolist()):              # what a masked slot holds does not matter
            for i in range(m):
                for h in range(K):
                    if float(bias[b, h, i]) == -INF:
                        for x in views:
                            x[int(of[0][b, i // page]), h, i % page] = (math.nan, INF)[i % 2]
            bias[b, :, m:] = math.nan
        out.append(bias)
    gap = 0 if tokens is None else 2
    T = len(own) if tokens is None else sum(tokens) + 2 * gap
    q = (torch.randn(T, H, d, generator=gen) * 2).to(TYPES[dtype])
    q_offsets = None if tokens is None else Q.offsets_of(tokens, gap)
    cuts = None if groups is None else torch.tensor(groups, dtype=torch.int32)
    return q, q_offsets, kv, views, pre, cuts, mine, out


@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_shared_attention(bench, case):
    dtype, H, K, d, page, order = case[0], case[1], case[2], case[3], case[4], case[9]
    q, q_offsets, kv, views, pre, cuts, mine, bias = _shared_case(case, _gen(H * d + page))
    seven = torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0)
    want = Q.shared_reference(q, q_offsets, *views, page, pre, cuts, mine, d ** -0.5, *bias, *seven, dtype)
    got = Q.run_shared(bench, q, q_offsets, kv, order, pre, cuts, mine, d ** -0.5, *bias)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


def test_shared_attention_is_attention_of_one_token_over_the_whole(bench):
    """A prefix and own slots, and the same pages as one sequence through sttm_paged_attention."""
    gen, page, d = _gen(3), 16, 64
    kv, table = C.pool(gen, "f32", 2, d, page, (48, 21, 37))
    q = torch.randn(2, 6, d, generator=gen)
    own = (table[1:], torch.tensor([21, 37], dtype=torch.int32))
    got = Q.run_shared(bench, q, None, kv, "pages", (table[:1], torch.tensor([48], dtype=torch.int32)), torch.tensor([0, 2], dtype=torch.int32), own, 0.2)
    whole = torch.full((2, 8), -1, dtype=torch.int32)
    for b, n in enumerate((21, 37)):
        pages = torch.cat([table[0, :3], table[1 + b, :-(-n // page)]])
        whole[b, :len(pages)] = pages
    out, lse, _ = C.run_attention(bench, q, kv, "pages", whole, torch.tensor([69, 85], dtype=torch.int32), 0.2)
    close(got[0], out.double().cpu(), 64 * C.E * 8, what="out")
    close(got[1], lse.double().cpu(), 64 * C.E * 8, what="lse")


def test_shared_attention_with_pages_outside_of_the_pool(bench):
    """Their slots count as masked: in a prefix, all over one, and among a sequence's own."""
    gen, page = _gen(5), 8
    kv, table = C.pool(gen, "bf16", 2, 64, page, (61, 40, 30, 90, 20))
    table[0, 2], table[0, 5], table[0, 7] = -1, kv[0].shape[0], 2 ** 31 - 1
    table[1, :5] = -1
    table[3, 1], table[3, 11] = -5, 10 ** 9
    pre = (table[:2].contiguous(), torch.tensor([61, 40], dtype=torch.int32))
    own = (table[2:].contiguous(), torch.tensor([30, 90, 20], dtype=torch.int32))
    cuts, q_offsets = torch.tensor([0, 1, 3], dtype=torch.int32), Q.offsets_of((2, 90, 1))
    q = torch.randn(93, 4, 64, generator=gen).to(torch.bfloat16)
    seven = torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0)
    want = Q.shared_reference(q, q_offsets, *kv, page, pre, cuts, own, 0.125, None, None, *seven, "bf16")
    got = Q.run_shared(bench, q, q_offsets, kv, "pages", pre, cuts, own, 0.125)
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


@pytest.mark.parametrize("dtype,d,tokens", [("bf16", 64, 70), ("f16", 136, 33), ("f32", 40, 66), ("f32", 256, 33), ("bf16", 32, 9), ("f16", 24, 12)])
@pytest.mark.parametrize("heads", [1, 3])
def test_shared_attention_of_values_that_later_tokens_see(bench, dtype, d, tokens, heads):
    """What a slot holds that a token does not see yet does not matter to it: infinite and NaN values and keys of the newest tokens;
    the tokens that see a value get it."""
    gen, page, n = _gen(d), 8, tokens + 60
    kv, table = C.pool(gen, dtype, 1, d, page, (19, n))
    pre, own = (table[:1].contiguous(), torch.tensor([19], dtype=torch.int32)), (table[1:].contiguous(), torch.tensor([n], dtype=torch.int32))
    for i, channel, value in ((n - 3, 3, INF), (n - 2, 5, math.nan), (n - 9, 7, -INF), (n - 8, 7, INF), (60 + tokens // 2, 1, INF), (2, 9, -INF)):
        kv[1][int(own[0][0, i // page]), 0, i % page, channel] = value
    kv[0][int(own[0][0, (n - 1) // page]), 0, (n - 1) % page, 4] = math.nan
    q = torch.randn(tokens, heads, d, generator=gen).to(TYPES[dtype])
    seven, cuts = (torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0)), torch.tensor([0, 1], dtype=torch.int32)
    want = Q.shared_reference(q, Q.offsets_of((tokens,)), *kv, page, pre, cuts, own, 0.1, None, None, *seven, dtype)
    got = Q.run_shared(bench, q, Q.offsets_of((tokens,)), kv, "pages", pre, cuts, own, 0.1)
    assert torch.isfinite(want[0][0][0, :, 3]).all() and torch.isinf(want[0][0][-2, :, 3]).all() and torch.isnan(want[0][0][-1]).all()
    close(got[0], *want[0], what="out")
    close(got[1], *want[1], what="lse")


def test_shared_attention_of_groups_with_offsets_that_make_no_sense(bench):
    """Whatever the tables hold, reads and writes stay inside: lengths below zero and beyond the tables, groups beyond the batch."""
    gen, page = _gen(8), 8
    kv, table = C.pool(gen, "bf16", 1, 32, page, (30, 20, 25), junk=0.0)
    table = table.clamp(0, kv[0].shape[0] - 1)
    q = torch.randn(5, 2, 32, generator=gen).to(torch.bfloat16)
    for lengths, groups, offsets in (((10 ** 9, -4), (0, 7), (0, 2, 5)), ((20, 25), (5, 1), (4, 2, 9)), ((20, 25), (-3, 2), (-7, 3, 10 ** 15)),
                                     ((20, 25), (1, 1), (5, 5, 5))):
        out, lse = Q.run_shared(bench, q, torch.tensor(offsets), kv, "pages", (table[:1], torch.tensor([30], dtype=torch.int32)),
                                torch.tensor(groups, dtype=torch.int32), (table[1:], torch.tensor(lengths, dtype=torch.int32)), 0.3)
        assert out.shape == q.shape


@pytest.mark.parametrize("dtype,tokens,n", [("bf16", 1, 70), ("f16", 40, 1100), ("f32", 2, 1100), ("f32", 70, 90)])
def test_results_in_the_place_of_the_queries(bench, dtype, tokens, n):
    """With one part a row and with several, few rows and many, against the call with a place of its own."""
    gen, lib, page, d, H, K = _gen(n), bench.lib, 64, 32, 4, 2
    storage, view = Q.states(gen, dtype, K, d, n, "projection")
    kv, table = C.pool(gen, dtype, K, d, page, (n, tokens + 3))
    q, q_offsets = torch.randn(tokens, H, d, generator=gen).to(TYPES[dtype]), bench.put(Q.offsets_of((tokens,)))
    st = lib.States(*view([bench.put(x) for x in storage]), bench.put(Q.offsets_of((n,))))
    cache, groups = lib.PagedCache(*[bench.put(x) for x in kv]), bench.put(torch.tensor([0, 1], dtype=torch.int32))
    pre, own = (lib.Sequences(bench.put(table[i:i + 1]), bench.put(torch.tensor([m], dtype=torch.int32))) for i, m in enumerate((n, tokens + 3)))
    ws = bench.workspace(max(lib.sttm_cross_attention_workspace_bytes(st, tokens, H), lib.sttm_shared_attention_workspace_bytes(cache, pre, own, tokens, H)))
    calls = (lambda x, o: bench.ctx.sttm_cross_attention(x, st, o, 0.2, q_offsets=q_offsets, workspace=ws),
             lambda x, o: bench.ctx.sttm_shared_attention(x, cache, pre, groups, own, o, 0.2, q_offsets=q_offsets, workspace=ws))
    for call in calls:
        apart, both = bench.guarded(torch.zeros_like(q)), bench.guarded(q)
        call(bench.put(q), apart)
        call(both, both)
        bench.done()
        assert torch.equal(apart, both)


# -- refusals ----------------------------------------------------------------------------------------------------------

def _refused(bench, code, call, *args, **kw):
    with pytest.raises(bench.lib.SttmError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_refusals_of_cross_attention(bench):
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    off = bench.put(torch.tensor([0, 3, 5]))
    _refused(bench, lib.STTM_ERR_SHAPE, lib.States, z(5, 2, 16), z(5, 2, 24), off)
    _refused(bench, lib.STTM_ERR_SHAPE, lib.States, z(5, 16, 2).transpose(1, 2), z(5, 16, 2).transpose(1, 2), off)
    _refused(bench, lib.STTM_ERR_DTYPE, lib.States, z(5, 2, 16), z(5, 2, 16).half(), off)
    _refused(bench, lib.STTM_ERR_DTYPE, lib.States, z(5, 2, 16), z(5, 2, 16), off.int())
    _refused(bench, lib.STTM_ERR_SHAPE, lib.States, z(5, 2, 16), z(5, 2, 16), off[:, None])
    _refused(bench, lib.STTM_ERR_SHAPE, lib.States, z(5, 2, 16), z(5, 2, 16), off, -1)
    for shape in ((5, 2, 12), (5, 2, 264), (5, 1025, 8)):
        st = lib.States(z(*shape), z(*shape), off)
        assert lib.sttm_cross_attention_workspace_bytes(st, 2, shape[1]) == 0
        _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, z(2, shape[1], shape[2]), st, z(2, shape[1], shape[2]), 1.0)
    odd = z(5 * 2 * 16 + 1)[1:].view(5, 2, 16)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_cross_attention, z(2, 2, 16), lib.States(odd, odd, off), z(2, 2, 16), 1.0)
    wide = z(5, 2, 18)[..., :16]
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, z(2, 2, 16), lib.States(wide, wide, off), z(2, 2, 16), 1.0)
    st = lib.States(z(5, 2, 16), z(5, 2, 16), off)
    ws = bench.workspace(1 << 16)
    q, ok = z(2, 4, 16), dict(workspace=ws)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0)
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, workspace=ws[:128])
    _refused(bench, lib.STTM_ERR_WORKSPACE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, workspace=ws[1:])
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, z(3, 4, 16), st, z(3, 4, 16), 1.0, **ok)        # three tokens of two sequences
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, z(2, 3, 16), st, z(2, 3, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, z(2, 514, 16), st, z(2, 514, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 24), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, ctx.sttm_cross_attention, q.half(), st, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, key_bias=z(4), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, key_bias=z(4, 5), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, key_bias=z(5, 2).T, **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, key_bias=z(5).half(), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, q_offsets=off[:2], **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, q_offsets=off.int(), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, lse=z(2, 3), **ok)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_cross_attention, q, st, z(2, 4, 16), math.nan, **ok)
    _refused(bench, lib.STTM_ERR_ARG, ctx.sttm_cross_attention, q, st, z(2, 4, 16), INF, **ok)
    st.struct.rows = (1 << 40) + 1                                # (described only)
    assert lib.sttm_cross_attention_workspace_bytes(st, 2, 4) == 0
    st.struct.rows, st.struct.row_stride = 1 << 40, 1 << 30
    _refused(bench, lib.STTM_ERR_SHAPE, ctx.sttm_cross_attention, q, st, z(2, 4, 16), 1.0, **ok)
    assert lib.sttm_cross_attention_workspace_bytes(lib.States(z(5, 2, 16), z(5, 2, 16), off), (1 << 22) + 1, 4) == 0
    bench.done()


def test_refusals_of_shared_attention(bench):
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    i = lambda *s: z(*s, dtype=torch.int32)   # noqa: E731
    cache = lib.PagedCache(z(4, 2, 8, 16), z(4, 2, 8, 16))
    pre, seqs, cuts, q = lib.Sequences(i(1, 2), i(1)), lib.Sequences(i(2, 2), i(2)), i(2), z(2, 4, 16)
    ws = bench.workspace(1 << 16)
    call, ok = ctx.sttm_shared_attention, dict(workspace=ws)
    _refused(bench, lib.STTM_ERR_WORKSPACE, call, q, cache, pre, cuts, seqs, z(2, 4, 16), 1.0)
    _refused(bench, lib.STTM_ERR_ARG, call, q, cache, pre, None, seqs, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_ARG, call, q, cache, None, cuts, seqs, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_ARG, call, q, cache, None, None, seqs, z(2, 4, 16), 1.0, prefix_bias=z(1, 2, 16), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, cache, pre, i(3), seqs, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, z(3, 4, 16), cache, pre, cuts, seqs, z(3, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, z(2, 3, 16), cache, pre, cuts, seqs, z(2, 3, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, cache, pre, cuts, seqs, z(2, 4, 16), 1.0, prefix_bias=z(1, 2, 15), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, cache, pre, cuts, seqs, z(2, 4, 16), 1.0, key_bias=z(2, 2, 15), **ok)
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, cache, pre, cuts, seqs, z(2, 4, 16), 1.0, key_bias=z(1, 2, 16), **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, call, q.half(), cache, pre, cuts, seqs, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_DTYPE, call, q, cache, pre, cuts.long(), seqs, z(2, 4, 16), 1.0, **ok)
    _refused(bench, lib.STTM_ERR_ARG, call, q, cache, pre, cuts, seqs, z(2, 4, 16), -INF, **ok)
    bad = lib.PagedCache(z(2, 2, 4, 16), z(2, 2, 4, 16))
    assert lib.sttm_shared_attention_workspace_bytes(bad, pre, seqs, 2, 4) == 0
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, bad, pre, cuts, seqs, z(2, 4, 16), 1.0, **ok)
    pre.struct.max_pages = pre.struct.table_stride = 1 << 28       # (described only)
    assert lib.sttm_shared_attention_workspace_bytes(cache, pre, seqs, 2, 4) == 0
    _refused(bench, lib.STTM_ERR_SHAPE, call, q, cache, pre, cuts, seqs, z(2, 4, 16), 1.0, **ok)
    bench.done()


def test_nothing_to_do(bench):
    """No tokens, no sequences: no launch, no error, nothing written."""
    lib, ctx = bench.lib, bench.ctx
    z = lambda *s, dtype=torch.float32: bench.put(torch.zeros(*s, dtype=dtype))   # noqa: E731
    st = lib.States(z(5, 2, 16), z(5, 2, 16), bench.put(torch.tensor([0])))
    ctx.sttm_cross_attention(z(0, 4, 16), st, z(0, 4, 16), 1.0)
    out = bench.guarded(torch.full((3, 4, 16), 7.0))
    ctx.sttm_cross_attention(z(3, 4, 16), st, out, 1.0, q_offsets=bench.put(torch.tensor([0])))
    cache = lib.PagedCache(z(2, 2, 8, 16), z(2, 2, 8, 16))
    none = lib.Sequences(z(0, 2, dtype=torch.int32), z(0, dtype=torch.int32))
    ctx.sttm_shared_attention(z(3, 4, 16), cache, None, None, none, out, 1.0, q_offsets=bench.put(torch.tensor([0])))
    bench.done()
    assert (out == 7).all()
