"""What the tests of the attention of several queries share: the definitions in 64 bits and calls through the binding, on the
`Bench` and the pools of cache_cases.

Tolerances, derived before the first run. u: the result type's rounding (bf16 2^-8, fp16 2^-11, fp32 2^-24); e = 2^-24.
* a score s = scale q.k + bias: D = (d + 4) e (scale sum |q_i k_i| + |bias|).
* a softmax weight is off by a factor of 1 + 2 D, the sums of n of them by n e, exponentials and the joining of parts by 64 e; 16-bit
  types round it once more before it meets a value: u, and in fp16, which holds 2^15 times the weight, 2^-40 of the largest weight
  where exponents run out.
* the result's own rounding: u.
"""
import torch

from tests.cache_cases import E, INF, TYPES, U, cache_views

LEAST = {"f32": 2.0 ** -140, "bf16": 2.0 ** -140, "f16": 2.0 ** -25}


def attend(q, k, v, scale, bias, seen, dtype):
    """Rows q [m, d] over keys k [n, d], those of row i that seen[i] (bool [n]) says: (out, its tolerance, lse, its tolerance)."""
    q, k, v = q.double(), k.double(), v.double()
    m, d = q.shape
    out, lse = torch.zeros(m, v.shape[1], dtype=torch.float64), torch.full((m,), -INF, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(m):
        at = seen[i] if bias is None else seen[i] & (bias != -INF)
        if not at.any():
            continue
        kk, vv = k[at], v[at]
        x, D = (kk * q[i]).sum(1) * scale, (kk * q[i]).abs().sum(1) * abs(scale)
        if bias is not None:
            x, D = x + bias[at].double(), D + bias[at].double().abs()
        D = D * (d + 4) * E
        D = float(torch.nan_to_num(torch.where(D > 1e30, 0.0, D)).max())
        n, top = int(at.sum()), x.max()
        p = torch.exp(x - top)
        total = p.sum()
        p = p / total
        lse[i] = top + torch.log(total)
        lse_tol[i] = D + (n + 64) * E + 4 * E * abs(float(top))
        out[i] = p @ vv
        rounded = 0.0 if dtype == "f32" else U[dtype]
        out_tol[i] = (p @ vv.abs()) * (2 * D + (n + 64) * E + rounded) + (2.0 ** -40 * vv.abs().sum(0) if dtype == "f16" else 0)
    return out, out_tol + U[dtype] * (1 + 2 ** -6) * out.abs() + LEAST[dtype], lse, lse_tol


# -- packed states -----------------------------------------------------------------------------------------------------

def offsets_of(lengths, first=0):
    x = [first]
    for n in lengths:
        x.append(x[-1] + n)
    return torch.tensor(x, dtype=torch.int64)


def states(gen, dtype, K, d, rows, layout, junk=float("nan")):
    """The storage behind k and v, and how to look at it (the same for copies): "projection" keys and values of one row side by
    side, "heads" a block for each head, "gap" rows that lie further apart."""
    t = TYPES[dtype]
    if layout == "projection":
        x = torch.randn(rows, 2 * K, d, generator=gen).to(t)
        return [x], lambda s: (s[0][:, :K], s[0][:, K:])
    if layout == "heads":
        x = [torch.randn(K, rows, d, generator=gen).to(t) for _ in range(2)]
        return x, lambda s: (s[0].transpose(0, 1), s[1].transpose(0, 1))
    x = [torch.full((rows, K, d + 16), junk, dtype=t) for _ in range(2)]
    for y in x:
        y[..., :d] = torch.randn(rows, K, d, generator=gen).to(t)
    return x, lambda s: (s[0][..., :d], s[1][..., :d])


def cross_reference(q, q_offsets, k, v, offsets, scale, bias, out, lse, dtype, max_rows=None):
    """(out, tolerance), (lse, tolerance); rows of no sequence as they were in out and lse."""
    T, H, d = q.shape
    K = k.shape[1]
    o, ot, l, lt = out.double().clone(), torch.zeros(T, H, d, dtype=torch.float64), lse.double().clone(), torch.zeros(T, H, dtype=torch.float64)
    for b in range(len(offsets) - 1):
        a0, a1 = (b, b + 1) if q_offsets is None else (int(q_offsets[b]), int(q_offsets[b + 1]))
        k0, k1 = int(offsets[b]), int(offsets[b + 1])
        if max_rows is not None:
            k1 = min(k1, k0 + max_rows)
        for h in range(H if a1 > a0 else 0):
            g = h // (H // K)
            add = None if bias is None else (bias if bias.dim() == 1 else bias[g])[k0:k1]
            seen = torch.ones(a1 - a0, k1 - k0, dtype=torch.bool)
            o[a0:a1, h], ot[a0:a1, h], l[a0:a1, h], lt[a0:a1, h] = attend(q[a0:a1, h], k[k0:k1, g], v[k0:k1, g], scale, add, seen, dtype)
    return (o, ot), (l, lt)


def run_cross(bench, q, q_offsets, storage, view, offsets, scale, bias=None, max_rows=None):
    lib = bench.lib
    k, v = view([bench.put(x) for x in storage])
    st = lib.States(k, v, bench.put(offsets), max_rows)
    out, lse = bench.guarded(torch.full_like(q, 7.0)), bench.guarded(torch.full(q.shape[:2], 7.0))
    need = lib.sttm_cross_attention_workspace_bytes(st, q.shape[0], q.shape[1])
    assert need >= 256
    bench.ctx.sttm_cross_attention(bench.put(q), st, out, scale, q_offsets=bench.put(q_offsets), key_bias=bench.put(bias), lse=lse,
                                   workspace=bench.workspace(need))
    bench.done()
    return out, lse


# -- a shared prefix ---------------------------------------------------------------------------------------------------

def gathered(x, table, n, page):
    """Slots of one sequence, [n, kv_heads, d], and which of them are in the pool."""
    at = [int(table[i // page]) for i in range(n)]
    ok = torch.tensor([0 <= p < x.shape[0] for p in at], dtype=torch.bool)
    rows = [x[p, :, i % page] if 0 <= p < x.shape[0] else torch.zeros_like(x[0, :, 0]) for i, p in enumerate(at)]
    return torch.stack(rows) if rows else x.new_zeros(0, x.shape[1], x.shape[3]), ok


def shared_reference(q, q_offsets, k, v, page, prefixes, groups, own, scale, prefix_bias, key_bias, out, lse, dtype):
    """prefixes, own: (table, lengths), prefixes None: none."""
    T, H, d = q.shape
    K = k.shape[1]
    o, ot, l, lt = out.double().clone(), torch.zeros(T, H, d, dtype=torch.float64), lse.double().clone(), torch.zeros(T, H, dtype=torch.float64)
    table, lengths = own
    for b in range(len(lengths)):
        a0, a1 = (b, b + 1) if q_offsets is None else (int(q_offsets[b]), int(q_offsets[b + 1]))
        m, n = a1 - a0, min(max(int(lengths[b]), 0), table.shape[1] * page)
        kk, ok = gathered(k, table[b], n, page)
        vv, _ = gathered(v, table[b], n, page)
        add = key_bias[b, :, :n] if key_bias is not None else torch.zeros(K, n)
        seen = torch.arange(n) < (n - m + 1 + torch.arange(m))[:, None]
        seen = seen & ok
        mine = [g for g in range(len(groups) - 1) if int(groups[g]) <= b < int(groups[g + 1])] if prefixes is not None else []
        if mine:
            g = mine[0]
            p = min(max(int(prefixes[1][g]), 0), prefixes[0].shape[1] * page)
            pk, pok = gathered(k, prefixes[0][g], p, page)
            pv, _ = gathered(v, prefixes[0][g], p, page)
            kk, vv = torch.cat([pk, kk]), torch.cat([pv, vv])
            add = torch.cat([prefix_bias[g, :, :p] if prefix_bias is not None else torch.zeros(K, p), add], 1)
            seen = torch.cat([pok.expand(m, p), seen], 1)
        for h in range(H if m > 0 else 0):
            c = h // (H // K)
            o[a0:a1, h], ot[a0:a1, h], l[a0:a1, h], lt[a0:a1, h] = attend(q[a0:a1, h], kk[:, c], vv[:, c], scale, add[c], seen, dtype)
    return (o, ot), (l, lt)


def run_shared(bench, q, q_offsets, kv, order, prefixes, groups, own, scale, prefix_bias=None, key_bias=None, lens=(None, None)):
    lib, d = bench.lib, q.shape[-1]
    cache = lib.PagedCache(*cache_views([bench.put(x) for x in kv], order, d))

    def limit(given, of, bias):                              # (a bias has no room for all slots of the table)
        return given if given is not None or bias is None else max([0] + [int(x) for x in of[1]])

    pre = None if prefixes is None else lib.Sequences(bench.put(prefixes[0]), bench.put(prefixes[1]), limit(lens[0], prefixes, prefix_bias))
    seqs = lib.Sequences(bench.put(own[0]), bench.put(own[1]), limit(lens[1], own, key_bias))
    out, lse = bench.guarded(torch.full_like(q, 7.0)), bench.guarded(torch.full(q.shape[:2], 7.0))
    need = lib.sttm_shared_attention_workspace_bytes(cache, pre, seqs, q.shape[0], q.shape[1])
    assert need >= 256
    bench.ctx.sttm_shared_attention(bench.put(q), cache, pre, None if pre is None else bench.put(groups), seqs, out, scale, q_offsets=bench.put(q_offsets),
                                    prefix_bias=bench.put(prefix_bias), key_bias=bench.put(key_bias), lse=lse, workspace=bench.workspace(need))
    bench.done()
    return out, lse
