"""The operators behind the merge, on a paged key-value cache: cases for timing them and for comparing their results.

Three operators, each one call of the ctypes binding:

* "rope":      queries and keys of a fused projection normalised per head and rotated by their positions, keys and values
               put into their slots of the cache (`sttm_qk_norm_rope`);
* "attention": one new token of every sequence attends to its cached keys; optionally with a bias per key (a merged token
               stands for several cells: the log of its count) and with the weight of every key added up
               (`sttm_paged_attention`);
* "evict":     of every sequence and key-value head the slots with the most accumulated weight stay, the survivors behind
               the new length fill the holes before it (`sttm_cache_evict`).

`run` has each of them in plain form too: elementary torch operations in 32 bits, rounded once at the end.
"""
import functools
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
THETA = 1e6
GAP = 1 << 40            # between protected slots, slots with a weight, and the rest


def _case(name, **c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # -- one token of one answer: a 7B model of 3584 channels (28 heads of 128, 4 for keys and values), launch and latency
        _case("rope_one_token", kind="rope", n=1, q_heads=28, kv_heads=4, d=128, dtype="bf16", page=16, norm=True, rotated=128,
              positions="index", interleaved=False),
        # one token for each of 48 answers, 8192 channels (64 heads of 128, 8 for keys and values), no norm
        _case("rope_step_of_48", kind="rope", n=48, q_heads=64, kv_heads=8, d=128, dtype="bf16", page=32, norm=False,
              rotated=128, positions="index", interleaved=False),
        # the prefill of the long video (512 frames of 13 x 13) reduced to half, positions (t, y, x) of the roots
        _case("rope_long_video_half", kind="rope", n=43264, q_heads=28, kv_heads=4, d=128, dtype="bf16", page=16, norm=True,
              rotated=128, positions="grid", interleaved=False),
        # rows of 1152 channels in 16 heads of 72, 30 % of 64 frames of 16 x 16, fractional positions of merged tokens,
        # neighbouring channels paired, the last 8 of a head left as they are
        _case("rope_merged_positions_f32", kind="rope", n=4915, q_heads=16, kv_heads=16, d=72, dtype="f32", page=16, norm=True,
              rotated=64, positions="merged", interleaved=True),
        # -- the answer to a short prompt: one sequence, few keys
        _case("attention_short", kind="attention", B=1, shortest=257, longest=257, q_heads=28, kv_heads=4, d=128, dtype="bf16",
              page=16, bias="", weights=False),
        # the answer about the long video reduced to half, every key's weight added up
        _case("attention_long_video_half", kind="attention", B=1, shortest=43328, longest=43328, q_heads=28, kv_heads=4, d=128,
              dtype="bf16", page=16, bias="", weights=True),
        # a batch of a larger model's answers, from short clips to long videos
        _case("attention_ragged_batch", kind="attention", B=24, shortest=901, longest=25977, q_heads=64, kv_heads=8, d=128,
              dtype="bf16", page=32, bias="", weights=False),
        # full precision, heads of 72 without groups, keys weighted by how many cells they stand for, some masked, and one
        # sequence whose keys all are
        _case("attention_counts_f32", kind="attention", B=5, shortest=333, longest=4979, q_heads=16, kv_heads=16, d=72,
              dtype="f32", page=16, bias="counts", weights=True),
        # -- a full cache takes one more token: one slot of each head goes
        _case("evict_one_each", kind="evict", B=16, shortest=4097, longest=4097, kept=4096, share=0.0, kv_heads=8, d=128,
              dtype="bf16", page=16, sink=4, recent=64, bias=False, again=True),
        # after the prefill of the long video, half of the cache goes
        _case("evict_long_video_half", kind="evict", B=1, shortest=43328, longest=43328, kept=0, share=0.5, kv_heads=4, d=128,
              dtype="bf16", page=16, sink=4, recent=64, bias=False, again=False),
        # a ragged batch with counts to 30 %
        _case("evict_ragged_batch", kind="evict", B=24, shortest=901, longest=25977, kept=0, share=0.3, kv_heads=8, d=128,
              dtype="bf16", page=32, sink=16, recent=128, bias=True, again=True),
        # few slots of full precision
        _case("evict_small_f32", kind="evict", B=3, shortest=131, longest=1013, kept=0, share=0.7, kv_heads=16, d=72,
              dtype="f32", page=16, sink=1, recent=17, bias=True, again=False),
    ]


LAYOUTS = [(28, 4, 128), (64, 8, 128), (16, 16, 72), (16, 2, 80), (14, 2, 64), (12, 4, 96), (10, 5, 256), (9, 3, 40), (16, 1, 128)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: every operator, type and head layout, from one token to the largest listed case."""
    kind = rng.choice(["rope", "attention", "evict"])
    q_heads, kv_heads, d = rng.choice(LAYOUTS)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    page = rng.choice([8, 16, 16, 32, 64])
    width = 4 if dtype == "f32" else 2
    if kind == "rope":
        row = (q_heads + 2 * kv_heads) * d * width
        n = min(_log_int(rng, 1, 43264), int(390e6 / row))
        return _case("", kind=kind, n=n, q_heads=q_heads, kv_heads=kv_heads, d=d, dtype=dtype, page=page, norm=rng.random() < 0.6,
                     rotated=rng.choice([d, d, d // 16 * 8]), positions=rng.choice(["index", "grid", "merged"]),
                     interleaved=rng.random() < 0.3)
    B = _log_int(rng, 1, 48)
    longest = _log_int(rng, 1, 43328)
    shortest = max(1, int(longest * rng.choice([1.0, 1.0, 0.3, 0.05])))
    token = 2 * kv_heads * d * width
    while sum(_spread(B, shortest, longest)) * token > 700e6:
        B, longest = (B // 2, longest) if B > 1 else (B, longest // 2)
        shortest = min(shortest, longest)
    c = _case("", kind=kind, B=B, shortest=shortest, longest=longest, kv_heads=kv_heads, d=d, dtype=dtype, page=page)
    if kind == "attention":
        c.update(q_heads=q_heads, bias=rng.choice(["", "", "counts"]), weights=rng.random() < 0.5)
    else:
        one = rng.random() < 0.4
        c.update(kept=max(1, shortest - 1) if one else 0, share=0.0 if one else round(rng.uniform(0.1, 0.9), 2),
                 sink=rng.choice([0, 4, 16]), recent=rng.choice([0, 31, 64, 128]), bias=rng.random() < 0.5, again=rng.random() < 0.5)
    return c


# -- inputs -------------------------------------------------------------------------------------------------------------

def _spread(B, shortest, longest):
    """Lengths of B sequences, spread over their logarithm and not in their order."""
    n = [int(round(longest * (shortest / longest) ** (i / (B - 1)))) for i in range(B)] if B > 1 else [longest]
    return n[::2] + n[1::2][::-1]


def _keep(case, lengths):
    return [case["kept"] or max(1, int(n * case["share"])) for n in lengths]


def _pool(case, lengths, gen, filled=True):
    """A pool of pages for sequences of these lengths, keys and values in it, and which pages each sequence has (any)."""
    B, page, heads, d = len(lengths), case["page"], case["kv_heads"], case["d"]
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3
    k, v = (torch.zeros(pages, heads, page, d, dtype=TYPES[case["dtype"]], device=DEVICE) for _ in range(2))
    if filled:
        at = max(1, (1 << 24) // (heads * page * d))
        for i in range(0, pages, at):
            for x in (k, v):
                x[i:i + at] = torch.randn(x[i:i + at].shape, device=DEVICE, generator=gen)
    order = torch.randperm(pages, device=DEVICE, generator=gen).to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    return {"k": k, "v": v, "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device=DEVICE), "longest": max(lengths)}


def _positions(case, gen):
    n = case["n"]
    if case["positions"] == "index":                        # reassigned: the row's own index behind a prompt
        at = 37 if n > 64 else 21000
        return (torch.arange(n, dtype=torch.int32, device=DEVICE) + at)[:, None].contiguous()
    if case["positions"] == "merged":                       # the mean index of a merged token's cells: fractions
        return (torch.rand(n, 1, device=DEVICE, generator=gen) * 16384.0).sort(0).values
    root = torch.empty(n, 4, dtype=torch.int32, device=DEVICE)   # (t, y0, x0, level) of a token's root
    root[:, 0] = torch.arange(n, device=DEVICE) * 512 // n
    root[:, 1:3] = torch.randint(0, 13, (n, 2), device=DEVICE, generator=gen)
    root[:, 3] = 0
    return root


def _sections(case):
    pairs = case["rotated"] // 2
    if case["positions"] != "grid":
        return (pairs,)
    y = pairs * 3 // 8
    return (pairs - 2 * y, y, y)


def prepare(case, seed):
    torch.cuda.set_device(0)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, d = TYPES[case["dtype"]], case["d"]

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    if case["kind"] == "rope":
        n, q, kv = case["n"], case["q_heads"], case["kv_heads"]
        s = _pool(case, [n], gen, filled=False)
        t = torch.arange(n, device=DEVICE)
        qkv = torch.empty(n, (q + 2 * kv) * d, dtype=dtype, device=DEVICE)
        step = max(1, (1 << 24) // qkv.shape[1])
        for i in range(0, n, step):
            qkv[i:i + step] = normal(*qkv[i:i + step].shape)
        pairs = case["rotated"] // 2
        s.update(qkv=qkv, slots=s["table"][0].long()[t // case["page"]] * case["page"] + t % case["page"],
                 q_weight=(1 + 0.2 * normal(d)).to(dtype) if case["norm"] else None,
                 k_weight=(1 + 0.2 * normal(d)).to(dtype) if case["norm"] else None,
                 positions=_positions(case, gen), sections=_sections(case),
                 inv_freq=THETA ** (-torch.arange(pairs, device=DEVICE, dtype=torch.float32) / max(1, pairs)),
                 q_out=torch.zeros(n, q, d, dtype=dtype, device=DEVICE))
        return dict(s, case=case)
    lengths = _spread(case["B"], case["shortest"], case["longest"])
    s = _pool(case, lengths, gen)
    B, kv, cap = case["B"], case["kv_heads"], s["longest"]
    if case["kind"] == "attention":
        sharp = torch.rand(B, case["q_heads"], 1, device=DEVICE, generator=gen) * 3 + 0.3    # flat heads and pointed ones
        s.update(q=(normal(B, case["q_heads"], d) * sharp).to(dtype), scale=1 / math.sqrt(d), bias=None, weights_in=None,
                 weights_out=None, out=torch.zeros(B, case["q_heads"], d, dtype=dtype, device=DEVICE),
                 lse=torch.zeros(B, case["q_heads"], device=DEVICE))
        if case["bias"]:
            s["bias"] = torch.exp(normal(B, kv, cap)).ceil().log()
            s["bias"][torch.rand(B, kv, cap, device=DEVICE, generator=gen) < 0.1] = -math.inf
            if B > 1:
                s["bias"][1] = -math.inf
        if case["weights"]:
            s.update(weights_in=normal(B, kv, cap).exp() * 0.01, weights_out=torch.zeros(B, kv, cap, device=DEVICE))
        return dict(s, case=case)
    weights = torch.exp(2 * normal(B, kv, cap))
    weights[torch.rand(B, kv, cap, device=DEVICE, generator=gen) < 0.05] = 0.0           # keys that nothing looked at
    total = list(lengths)
    ids = torch.full((B, kv, cap), -1, dtype=torch.int32, device=DEVICE)
    if case["again"]:                                       # slots went before: the first half holds other tokens in any order
        half, total = [n // 2 for n in lengths], [n + n // 3 for n in lengths]
        for b in range(B):
            some = torch.rand(kv, max(1, total[b] - lengths[b] + half[b]), device=DEVICE, generator=gen).argsort(1)
            ids[b, :, :half[b]] = some[:, :half[b]].to(torch.int32)
    s.update(weights_in=weights, ids_in=ids, weights_out=torch.zeros_like(weights), ids_out=torch.zeros_like(ids),
             total=torch.tensor(total, dtype=torch.int32, device=DEVICE),
             keep=torch.tensor(_keep(case, lengths), dtype=torch.int32, device=DEVICE),
             lengths_out=torch.zeros(B, dtype=torch.int32, device=DEVICE), bias_in=None, bias_out=None)
    if case["bias"]:
        s.update(bias_in=torch.exp(normal(B, kv, cap)).ceil().log(), bias_out=torch.zeros(B, kv, cap, device=DEVICE))
    return dict(s, case=case)


# -- the framework's calls -------------------------------------------------------------------------------------------------

@functools.lru_cache(None)
def _context():
    from paper_2507_07990_amd import binding as lib
    return lib, lib.Sttm(0)


def _plan(s):
    """What a program sets up once for its buffers: descriptions of the cache and the sequences, and a workspace."""
    lib, ctx = _context()
    if "plan" not in s:
        case, need = s["case"], 0
        p = {"cache": lib.PagedCache(s["k"], s["v"])}
        if case["kind"] == "rope":
            p["rope"] = lib.Rope(s["positions"], s["inv_freq"], s["sections"], interleaved=case["interleaved"])
        else:
            p["sequences"] = lib.Sequences(s["table"], s["lengths"], s["longest"])
        if case["kind"] == "attention":
            need = lib.sttm_paged_attention_workspace_bytes(p["cache"], p["sequences"], case["q_heads"], case["weights"])
        elif case["kind"] == "evict":
            need = lib.sttm_cache_evict_workspace_bytes(p["cache"], p["sequences"])
        p["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEVICE) if need else None
        s["plan"] = p
    return ctx, s["plan"]


def _own(s):
    case = s["case"]
    ctx, p = _plan(s)
    if case["kind"] == "rope":
        q, k, v = _heads(s)
        ctx.sttm_qk_norm_rope(q, k, v, s["q_out"], cache=p["cache"], slots=s["slots"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                              eps=EPS, rope=p["rope"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if case["kind"] == "attention":
        ctx.sttm_paged_attention(s["q"], p["cache"], p["sequences"], s["out"], s["scale"], key_bias=s["bias"], weights_in=s["weights_in"],
                                 weights_out=s["weights_out"], lse=s["lse"], workspace=p["workspace"])
        return {"out": s["out"], "lse": s["lse"], "weights": s["weights_out"]}
    ctx.sttm_cache_evict(p["cache"], p["sequences"], s["keep"], s["lengths_out"], s["weights_in"], s["weights_out"], s["ids_in"], s["ids_out"],
                         total=s["total"], sink=case["sink"], recent=case["recent"], bias_in=s["bias_in"], bias_out=s["bias_out"],
                         workspace=p["workspace"])
    return {"k": s["k"], "v": s["v"], "lengths": s["lengths_out"], "weights": s["weights_out"], "ids": s["ids_out"], "bias": s["bias_out"]}


# -- the plain forms -------------------------------------------------------------------------------------------------------

def _heads(s):
    case, x = s["case"], s["qkv"].view(s["qkv"].shape[0], -1, s["case"]["d"])
    q, kv = case["q_heads"], case["kv_heads"]
    return x[:, :q], x[:, q:q + kv], x[:, q + kv:]


def _halves(x):
    """A 32-bit number as the sum of two of 12 significant bits: products of such halves are exact."""
    hi = (x.view(torch.int32) & ~0xfff).view(torch.float32)
    return hi, x - hi


def _turn(x, y):
    """Two rotations, one after the other."""
    return x[0] * y[0] - x[1] * y[1], x[0] * y[1] + x[1] * y[0]


def _angles(s):
    """cos and sin of position times frequency: the product rounded to 32 bits would be off by more than the result, so it
    is taken as four exact products whose rotations follow each other."""
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=DEVICE), torch.tensor(s["sections"], device=DEVICE))
    p0, p1 = _halves(s["positions"].float()[:, axis])
    f0, f1 = _halves(s["inv_freq"])
    a = torch.stack([p0 * f0, p0 * f1, p1 * f0, p1 * f1])
    c, n = torch.cos(a), torch.sin(a)
    return _turn(_turn((c[0], n[0]), (c[1], n[1])), _turn((c[2], n[2]), (c[3], n[3])))


def _rotate(x, weight, angles, interleaved):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    cos, sin = angles[0][:, None], angles[1][:, None]
    pairs = cos.shape[-1]
    rest = x[..., 2 * pairs:]
    if interleaved:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, rest], -1)


def _plain_rope(s):
    case, (q, k, v), angles = s["case"], _heads(s), _angles(s)
    page, at = s["slots"] // case["page"], s["slots"] % case["page"]
    s["q_out"].copy_(_rotate(q, s["q_weight"], angles, case["interleaved"]))
    s["k"][page, :, at] = _rotate(k, s["k_weight"], angles, case["interleaved"]).to(s["k"].dtype)
    s["v"][page, :, at] = v
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _gather(x, table):
    """Every sequence's rows one after the other, [B, heads, slots, d]."""
    B, n = table.shape
    return x[table.clamp(min=0).long()].transpose(1, 2).reshape(B, x.shape[1], n * x.shape[2], x.shape[3])


def _plain_attention(s):
    case, n = s["case"], s["longest"]
    B, q_heads, kv, d = case["B"], case["q_heads"], case["kv_heads"], case["d"]
    valid = (torch.arange(n, device=DEVICE) < s["lengths"][:, None])[:, None]                # [B, 1, n]
    if s["bias"] is not None:
        valid = valid & (s["bias"] > -math.inf)
    valid = valid.expand(B, kv, n)
    k = torch.where(valid[..., None], _gather(s["k"], s["table"])[:, :, :n].float(), 0.0)
    x = torch.matmul(s["q"].float().view(B, kv, q_heads // kv, d), k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    if s["bias"] is not None:
        x = x + s["bias"][:, :, None]
    x = torch.where(valid[:, :, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    v = torch.where(valid[..., None], _gather(s["v"], s["table"])[:, :, :n].float(), 0.0)
    s["out"].copy_(torch.matmul(p, v).view(B, q_heads, d))
    s["lse"].copy_((top + torch.log(total)).view(B, q_heads))
    if case["weights"]:
        inside = torch.arange(n, device=DEVICE) < s["lengths"][:, None, None]
        s["weights_out"].copy_(torch.where(inside, s["weights_in"] + p.sum(2), s["weights_out"]))
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights_out"]}


def _plain_evict(s):
    case, n, w = s["case"], s["longest"], s["weights_in"]
    i = torch.arange(n, device=DEVICE)
    length, total = s["lengths"][:, None, None].long(), s["total"][:, None, None].long()
    new = torch.minimum(s["keep"][:, None, None].long(), length)
    ids = torch.where(s["ids_in"] < 0, total - length + i, s["ids_in"].long())
    bits = (w + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -1 - (bits & 0x7fffffff), bits)                           # as the weights themselves
    order = torch.where(torch.isnan(w), -GAP, order)
    order = torch.where((ids < case["sink"]) | (ids >= total - case["recent"]), GAP, order)
    order = torch.where(i < length, order, -2 * GAP)
    by = torch.sort((order << 20) - ids, dim=-1, descending=True).indices
    rank = torch.empty_like(by).scatter_(-1, by, i.expand_as(by))
    kept = (rank < new) & (i < length)
    dst = torch.nonzero(~kept & (i < new), as_tuple=True)                                    # in order of (b, head, slot), both:
    src = torch.nonzero(kept & (i >= new), as_tuple=True)                                    # the j-th of one goes to the j-th
    page = case["page"]
    to = (s["table"][dst[0], dst[2] // page].long(), dst[1], dst[2] % page)
    fro = (s["table"][src[0], src[2] // page].long(), src[1], src[2] % page)
    s["k"][to] = s["k"][fro]
    s["v"][to] = s["v"][fro]

    def table(given, out, rest):
        x = torch.where(i < new, given, rest)
        x[dst] = given[src]
        out.copy_(torch.where(i < length, x, out))

    table(w, s["weights_out"], 0.0)
    table(ids.to(torch.int32), s["ids_out"], -1)
    if case["bias"]:
        table(s["bias_in"], s["bias_out"], 0.0)
    s["lengths_out"].copy_(new.view(-1))
    return {"k": s["k"], "v": s["v"], "lengths": s["lengths_out"], "weights": s["weights_out"], "ids": s["ids_out"], "bias": s["bias_out"]}


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "attention": _plain_attention, "evict": _plain_evict}[state["case"]["kind"]](state)


# -- the definition in 64 bits -----------------------------------------------------------------------------------------------

def _exact_rope(s):
    case = s["case"]
    n, q, kv, d = case["n"], case["q_heads"], case["kv_heads"], case["d"]
    pairs = case["rotated"] // 2
    pos, freq = s["positions"].double(), s["inv_freq"].double()
    angle, at = [], 0
    for axis, width in enumerate(s["sections"]):
        angle.append(pos[:, axis, None] * freq[at:at + width])
        at += width
    z = torch.polar(torch.ones(n, pairs, dtype=torch.float64, device=DEVICE), torch.cat(angle, 1))

    def rows(lo, hi, weight):
        x = s["qkv"].double().view(n, -1, d)[:, lo:hi]
        if weight is not None:
            x = x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt() * weight.double()
        out = x.clone()
        for i in range(pairs):
            ia, ib = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs)
            r = torch.complex(x[..., ia].contiguous(), x[..., ib].contiguous()) * z[:, i, None]
            out[..., ia], out[..., ib] = r.real, r.imag
        return out

    k = s["k"].double()
    rotated = rows(q, q + kv, s["k_weight"])
    k[s["slots"] // case["page"], :, s["slots"] % case["page"]] = rotated
    return {"q": rows(0, q, s["q_weight"]), "k": k, "v": None}


def _exact_attention(s):
    case = s["case"]
    group, page = case["q_heads"] // case["kv_heads"], case["page"]
    out, lse = s["out"].double(), s["lse"].double()
    weights = s["weights_out"].double() if case["weights"] else None
    for b, n in enumerate(s["lengths"].tolist()):
        pages = s["table"][b, :-(-n // page)].long()
        for h in range(case["kv_heads"]):
            k, v = (x[pages, h].reshape(-1, case["d"])[:n].double() for x in (s["k"], s["v"]))
            for g in range(h * group, (h + 1) * group):
                x = (k * s["q"][b, g].double()).sum(1) * s["scale"]
                if s["bias"] is not None:
                    x = x + s["bias"][b, h, :n].double()
                lse[b, g] = torch.logsumexp(x, 0)
                p = torch.zeros_like(x) if torch.isneginf(lse[b, g]) else torch.exp(x - lse[b, g])
                out[b, g] = p @ v
                if weights is not None:
                    weights[b, h, :n] += p + (s["weights_in"][b, h, :n].double() if g == h * group else 0)
    return {"out": out, "lse": lse, "weights": weights}


def _exact_evict(s):
    """The numbers are moved, not computed: the weights alone, from a sort of each row on the host."""
    case = s["case"]
    weights, given, ids = s["weights_out"].double().cpu(), s["weights_in"].cpu(), s["ids_in"].cpu()
    for b, (n, total, keep) in enumerate(zip(s["lengths"].tolist(), s["total"].tolist(), s["keep"].tolist())):
        new = min(n, keep)
        for h in range(case["kv_heads"]):
            w = given[b, h, :n].tolist()
            name = [total - n + i if x < 0 else x for i, x in enumerate(ids[b, h, :n].tolist())]
            safe = [x < case["sink"] or x >= total - case["recent"] for x in name]
            stay = set(sorted(range(n), key=lambda i: (not safe[i], 0.0 if safe[i] else -w[i], name[i]))[:new])
            movers = iter([i for i in range(new, n) if i in stay])
            row = [w[i] if i in stay else w[next(movers)] for i in range(new)] + [0.0] * (n - new)
            weights[b, h, :n] = torch.tensor(row, dtype=torch.float64)
    return {"k": None, "v": None, "lengths": None, "weights": weights, "ids": None, "bias": None}


def exact(case, seed):
    if case["kind"] == "evict" and sum(_spread(case["B"], case["shortest"], case["longest"])) * case["kv_heads"] > 2_500_000:
        return None                                         # (a sort on the host: too long)
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attention": _exact_attention, "evict": _exact_evict}[case["kind"]](s)


# -- what cannot be done without -----------------------------------------------------------------------------------------------

def work(case):
    """rope: every row read once and written once, the positions read. attention: every cached key and value read once,
    queries, results and the tables by slot once. evict: the tables by slot read and written once, and the rows that fill
    the holes: of the slots before the new length those that go, as many as there would be if the weights knew no order."""
    width = 4 if case["dtype"] == "f32" else 2
    d, kv = case["d"], case["kv_heads"]
    if case["kind"] == "rope":
        row = (case["q_heads"] + 2 * kv) * d
        axes = {"index": 4, "merged": 4, "grid": 12}[case["positions"]]
        return {"bytes": case["n"] * (2 * row * width + 8 + axes), "flops": case["n"] * (case["q_heads"] + kv) * d * (7 if case["norm"] else 3)}
    lengths = _spread(case["B"], case["shortest"], case["longest"])
    cached = sum(lengths)
    if case["kind"] == "attention":
        slot = 2 * d * width + (4 if case["bias"] else 0) + (8 if case["weights"] else 0)
        return {"bytes": cached * kv * slot + case["B"] * case["q_heads"] * (2 * d * width + 4), "flops": 4.0 * cached * case["q_heads"] * d}
    moved = 0.0
    for n, keep in zip(lengths, _keep(case, lengths)):
        new, safe = min(n, keep), min(n, case["recent"]) + min(n, case["sink"])
        if new < n:
            stay = max(0.0, new - safe) / max(1, n - safe)
            moved += min(new, n - new, max(0, new - min(case["sink"], new)) * (1 - stay))
    tables = 4 if case["bias"] else 0
    return {"bytes": kv * (cached * 2 * (8 + tables) + moved * 4 * d * width), "flops": cached * kv}
