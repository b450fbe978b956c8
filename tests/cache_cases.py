"""What the tests of the operators on a paged cache share: inputs, the definitions in 64 bits, calls through the binding.

Everything here lives on the CPU; `Bench` moves it to the device of a context (the GPU, or host memory where the kernels are
built for host threads) and back, with a band of known bytes around every buffer that a call writes.

Tolerances, derived before the first run. u: the result type's rounding (bf16 2^-8, fp16 2^-11, fp32 2^-24); e = 2^-24.
* rotated rows: u |y| from the last rounding; the angle in half turns is rounded once (pi e) and sine and cosine are within a
  few ulps, so (|a| + |b|) 8 e; the mean of d squares, its root and the products ((d / 4 + 16) e |y|).
* a score s = scale q.k + bias: D = (d + 4) e (scale sum |q_i k_i| + |bias|).
* attention: a softmax weight is off by a factor of 1 + 2 D and the sums of n of them by n e, the exponentials by 4 e; in
  16 bits the weights are handed on as two numbers, 2^-16 (bf16) or 2^-21 and 2^-25 of the largest (fp16). An exponential
  below 2^-126, the smallest normal fp32 number, may be zero.
"""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SPLIT = {"f32": 0.0, "bf16": 2.0 ** -16, "f16": 2.0 ** -21}
E = 2.0 ** -24
BAND = 4096
INF = math.inf


class Bench:
    """A context, and buffers for it that are checked for writes outside."""

    def __init__(self, lib, ctx, device):
        self.lib, self.ctx, self.device, self.bands = lib, ctx, device, []

    def put(self, x):
        return None if x is None else x.to(self.device)

    def guarded(self, x):
        """A copy of x between two bands of known bytes."""
        n = x.numel() * x.element_size()
        raw = torch.full((n + 2 * BAND,), 0xA5, dtype=torch.uint8, device=self.device)
        raw[BAND:BAND + n] = x.contiguous().view(-1).view(torch.uint8).to(self.device) if n else raw[:0]
        self.bands.append((raw, n))
        return raw[BAND:BAND + n].view(x.dtype).view(x.shape)

    def workspace(self, n):
        """n bytes, 256-byte aligned, none of them zero (nothing may count on what they hold), bands around them."""
        raw = torch.full((n + 2 * BAND + 256,), 0xA5, dtype=torch.uint8, device=self.device)
        at = -(raw.data_ptr() + BAND) % 256
        raw = raw[at:at + n + 2 * BAND]
        raw[BAND:BAND + n] = 0xFF
        self.bands.append((raw, n))
        return raw[BAND:BAND + n]

    def done(self):
        if self.device != "cpu":
            torch.cuda.synchronize()
        for raw, n in self.bands:
            assert (raw[:BAND] == 0xA5).all() and (raw[BAND + n:] == 0xA5).all(), "bytes outside of a buffer were overwritten"
        self.bands = []


def close(got, want, tol, what=""):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(torch.where(inf, got, 0.0), torch.where(inf, want, 0.0)), f"{what}: infinities elsewhere"
    off = torch.where(torch.isfinite(want), (got - want).abs() - tol, -1.0)
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: {float(off.max())} over the tolerance"


# -- a pool of pages ---------------------------------------------------------------------------------------------------

def pool(gen, dtype, kv_heads, d, page, lengths, order="pages", junk=math.nan, spare=3):
    """k, v [pages, kv_heads, page, d] whose unused slots hold `junk`; a table whose unused entries name no page; order:
    "pages" (heads outside), "slots" (slots outside: the middle axes exchanged) or "padded" (every row further apart)."""
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    shape = (pages, page, kv_heads, d) if order == "slots" else (pages, kv_heads, page, d)
    if order == "padded":
        shape = shape[:3] + (d + 16,)
    kv = []
    for _ in range(2):
        x = torch.full(shape, junk, dtype=TYPES[dtype])
        kv.append(x)
    view = [x.transpose(1, 2) if order == "slots" else x[..., :d] for x in kv]
    table = torch.full((len(lengths), max(need + [1]) + 2), 10 ** 9, dtype=torch.int32)
    table[:, -1] = -7
    free = torch.randperm(pages, generator=gen).to(torch.int32)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :need[b]] = free[at:at + need[b]]
        at += need[b]
        for i in range(n):
            p = int(table[b, i // page])
            for x in view:
                x[p, :, i % page] = torch.randn(kv_heads, d, generator=gen).to(x.dtype)
    return kv, table


def cache_views(kv, order, d):
    return [x.transpose(1, 2) if order == "slots" else x[..., :d] for x in kv]


# -- norm and rotation -------------------------------------------------------------------------------------------------

def rope_reference(x, weight, eps, positions, inv_freq, sections, interleaved, u):
    """The rows in 64 bits, and how far a result of that type may be off."""
    x = x.double()
    d = x.shape[-1]
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    y, tol = x.clone(), torch.zeros_like(x)
    pair = 0
    for axis, width in enumerate(sections):
        for _ in range(width):
            angle = positions[:, axis].double() * float(inv_freq[pair])
            c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            ia, ib = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + sum(sections))
            y[..., ia] = x[..., ia] * c - x[..., ib] * s
            y[..., ib] = x[..., ia] * s + x[..., ib] * c
            tol[..., ia] = tol[..., ib] = (x[..., ia].abs() + x[..., ib].abs()) * 8 * E
            pair += 1
    if weight is not None:
        tol = tol + (d / 4 + 16) * E * (x.abs().amax(-1, keepdim=True) if sum(sections) else x.abs())
    return y, tol + u * y.abs() * (1 + 2 ** -6) + 2.0 ** -149 + (2.0 ** -25 if u == U["f16"] else 0)


# -- attention ---------------------------------------------------------------------------------------------------------

def attention_reference(q, k, v, table, lengths, page, scale, bias, weights_in, weights_out, dtype, max_len=None):
    """(result, tolerance) of out, lse and weights; k, v [pages, kv_heads, page, d]."""
    B, H, d = q.shape
    pages, kv_heads = k.shape[:2]
    group = H // kv_heads
    out, lse = torch.zeros(B, H, d, dtype=torch.float64), torch.full((B, H), -INF, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    weights = weights_out.double().clone() if weights_out is not None else None
    w_tol = torch.zeros_like(weights) if weights is not None else None
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * page if max_len is None else max_len)
        for h in range(kv_heads):
            slots = [i for i in range(n) if 0 <= int(table[b, i // page]) < pages and (bias is None or float(bias[b, h, i]) != -INF)]
            if weights is not None:
                weights[b, h, :n] = weights_in[b, h, :n].double() if weights_in is not None else 0.0
                w_tol[b, h, :n] = 2 * E * weights[b, h, :n].abs()
            if not slots:
                continue
            at = [int(table[b, i // page]) for i in slots]
            off = [i % page for i in slots]
            kk, vv = k[at, h, off].double(), v[at, h, off].double()
            for g in range(h * group, (h + 1) * group):
                qq = q[b, g].double()
                x, D = (kk * qq).sum(1) * scale, (kk * qq).abs().sum(1) * abs(scale)
                if bias is not None:
                    x = x + bias[b, h, slots].double()
                    D = D + bias[b, h, slots].double().abs()
                D = D * (d + 4) * E
                D = float(torch.nan_to_num(torch.where(D > 1e30, 0.0, D)).max())
                top = x.max()
                p = torch.exp(x - top)
                total = p.sum()
                p = p / total
                lse[b, g] = top + torch.log(total)
                lse_tol[b, g] = D + (n + 64) * E + 4 * E * abs(float(top))
                out[b, g] = p @ vv
                rel = 2 * D + (n + 64) * E
                out_tol[b, g] = (p @ vv.abs()) * (rel + SPLIT[dtype]) + (2.0 ** -24 * vv.abs().sum(0) if dtype == "f16" else 0)
                if weights is not None:
                    weights[b, h, slots] += p
                    w_tol[b, h, slots] += p * rel + E * weights[b, h, slots].abs() + 2.0 ** -126
    out_tol = out_tol + U[dtype] * (1 + 2 ** -6) * out.abs() + (2.0 ** -25 if dtype == "f16" else 2.0 ** -140)
    return (out, out_tol), (lse, lse_tol), (weights, w_tol)


def run_attention(bench, q, kv, order, table, lengths, scale, bias=None, weights_in=None, weights_out=None, max_len=None, alias=False):
    """The call on copies; returns out, lse and weights."""
    lib, d = bench.lib, q.shape[-1]
    k, v = cache_views([bench.put(x) for x in kv], order, d)
    cache = lib.PagedCache(k, v)
    if max_len is None and (bias is not None or weights_out is not None):   # (the tables have no room for the table's slots)
        max_len = int(lengths.max())
    seqs = lib.Sequences(bench.put(table), bench.put(lengths), max_len)
    qd = bench.put(q)
    out, lse = bench.guarded(torch.full_like(q, 7.0)), bench.guarded(torch.full(q.shape[:2], 7.0))
    bench_w = bench.guarded(weights_in if alias else weights_out) if weights_out is not None else None
    win = bench_w if alias else bench.put(weights_in)
    need = lib.sttm_paged_attention_workspace_bytes(cache, seqs, q.shape[1], weights_out is not None)
    assert need >= 256
    ws = bench.workspace(need)
    bench.ctx.sttm_paged_attention(qd, cache, seqs, out, scale, key_bias=bench.put(bias), weights_in=win, weights_out=bench_w,
                                   lse=lse, workspace=ws)
    bench.done()
    return out, lse, bench_w


# -- eviction ----------------------------------------------------------------------------------------------------------

def evict_reference(k, v, table, lengths, page, keep, total, sink, recent, weights, ids, bias, weights_out, ids_out, bias_out):
    """What the call leaves in k, v (as the views it gets) and the tables: lists of (slot <- slot) moves carried out one by one."""
    k, v = k.clone(), v.clone()
    pages, kv_heads = k.shape[:2]
    weights_out, ids_out = weights_out.clone(), ids_out.clone()
    bias_out = None if bias_out is None else bias_out.clone()
    new_lengths = []
    for b, n in enumerate(int(x) for x in lengths):
        tot = int(total[b]) if total is not None else n
        new = min(n, max(int(keep[b]), 0))
        new_lengths.append(new)
        for h in range(kv_heads):
            w = weights[b, h, :n].tolist()
            name = [tot - n + i if ids is None or int(ids[b, h, i]) < 0 else int(ids[b, h, i]) for i in range(n)]

            def order(i):
                safe = name[i] < sink or name[i] >= tot - recent
                if safe:
                    return (0, 0.0, name[i])
                if math.isnan(w[i]):
                    return (2, 0.0, name[i])
                return (1, -w[i], name[i])

            stay = sorted(range(n), key=order)[:new]
            holes = sorted(set(range(new)) - set(stay))
            movers = sorted(i for i in stay if i >= new)
            assert len(holes) == len(movers)
            weights_out[b, h, :new], weights_out[b, h, new:n] = weights[b, h, :new], 0.0
            ids_out[b, h, :new], ids_out[b, h, new:n] = torch.tensor(name[:new], dtype=torch.int32), -1
            if bias is not None:
                bias_out[b, h, :new], bias_out[b, h, new:n] = bias[b, h, :new], 0.0
            for to, fro in zip(holes, movers):
                weights_out[b, h, to], ids_out[b, h, to] = weights[b, h, fro], name[fro]
                if bias is not None:
                    bias_out[b, h, to] = bias[b, h, fro]
                p, r = int(table[b, to // page]), int(table[b, fro // page])
                if 0 <= p < pages and 0 <= r < pages:
                    k[p, h, to % page] = k[r, h, fro % page]
                    v[p, h, to % page] = v[r, h, fro % page]
    return k, v, weights_out, ids_out, bias_out, torch.tensor(new_lengths, dtype=torch.int32)


def run_evict(bench, kv, order, d, table, lengths, keep, total, sink, recent, weights, ids, bias, weights_out, ids_out, bias_out, alias=False):
    """The call on copies (alias: every output is its input); returns k, v, weights, ids, bias and lengths."""
    lib = bench.lib
    dev = [bench.guarded(x) for x in kv]
    cache = lib.PagedCache(*cache_views(dev, order, d))
    given = [bench.guarded(x) if x is not None else None for x in (weights, ids, bias)]
    outs = given if alias else [bench.guarded(x) if x is not None else None for x in (weights_out, ids_out, bias_out)]
    length = bench.guarded(lengths)
    new = length if alias else bench.guarded(torch.full_like(lengths, -3))
    seqs = lib.Sequences(bench.put(table), length, int(lengths.max()))
    ws = bench.workspace(lib.sttm_cache_evict_workspace_bytes(cache, seqs))
    bench.ctx.sttm_cache_evict(cache, seqs, bench.put(keep), new, given[0], outs[0], given[1], outs[1], total=bench.put(total), sink=sink,
                               recent=recent, bias_in=given[2], bias_out=outs[2], workspace=ws)
    bench.done()
    return (*cache_views(dev, order, d), *outs, new)
