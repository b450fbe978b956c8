"""A video's reduced tokens in one attention layer of a language model, from the merge to a cache that is reduced further.

    python examples/answer_from_reduced_video.py [--frames 64] [--keep 0.5] [--steps 32] [--cache-keep 0.5]

The layer's weights and the answer's tokens are random: this shows the calls in their order, not a model.

  1. merge: the video's tokens to a budget, with counts and position indices
  2. prefill: one projection for queries, keys and values; sttm_qk_norm_rope norms, rotates by the reassigned positions and
     puts keys and values into the pages of a cache; a merged token's keys get the log of its count as a bias
  3. answer: token by token, rotation and cache write, then sttm_paged_attention, which adds every key's weight up
  4. when the cache is full, sttm_cache_evict keeps the slots that were looked at most
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2507_07990_amd import binding as lib  # noqa: E402
from paper_2507_07990_amd import workloads as wl  # noqa: E402

PAGE, HEAD_DIM = 16, 128


def merge(ctx, feats, keep):
    """The reduced rows [n, D] of one video, how many tokens each stands for, and its index in the new sequence."""
    B, T, H, W, D = feats.shape
    N, dev = B * T * H * W, feats.device
    ctx.ensure_workspace(B, T, H, W, D, lib.STTM_BF16)
    ints = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device=dev)  # noqa: E731
    node_map, level, cluster = ints(N), ints(N, dtype=torch.uint8), ints(N)
    rows, counts, ids, offsets = torch.empty(N, D, dtype=feats.dtype, device=dev), ints(N), ints(N), ints(B + 1, dtype=torch.int64)
    index = ints(N)
    ctx.sttm_spatial_stats(feats, lib.STTM_BF16, B, T, H, W, D)
    ctx.sttm_budget_threshold(lib.STTM_STAGE_SPATIAL, keep, want_tau=False)
    ctx.sttm_spatial_quadtree(feats, lib.STTM_BF16, B, T, H, W, D, 1, None, node_map, level)
    ctx.sttm_temporal_stats(feats, node_map, level)
    ctx.sttm_budget_threshold(lib.STTM_STAGE_TEMPORAL, keep, want_tau=False)
    ctx.sttm_temporal_merge(feats, node_map, level, None, cluster)
    n = ctx.sttm_reduce(feats, cluster, node_map, level, lib.STTM_BF16, N, rows, counts, ids, offsets)
    ctx.sttm_positions(cluster, node_map, level, offsets, N, reassigned=index)
    return rows[:n], counts[:n], index[:n]


class Layer:
    """Queries, keys and values of one attention layer, and the cache behind it (one sequence)."""

    def __init__(self, ctx, width, q_heads, kv_heads, slots, dev, seed=0):
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.ctx, self.q_heads, self.kv_heads = ctx, q_heads, kv_heads
        heads = q_heads + 2 * kv_heads
        self.weight = (torch.randn(width, heads * HEAD_DIM, device=dev, generator=gen) / math.sqrt(width)).to(torch.bfloat16)
        self.q_norm = torch.ones(HEAD_DIM, dtype=torch.bfloat16, device=dev)
        self.k_norm = torch.ones(HEAD_DIM, dtype=torch.bfloat16, device=dev)
        self.inv_freq = 1e6 ** (-torch.arange(HEAD_DIM // 2, device=dev, dtype=torch.float32) / (HEAD_DIM // 2))
        pages = -(-slots // PAGE)
        kv = torch.zeros(2, pages, kv_heads, PAGE, HEAD_DIM, dtype=torch.bfloat16, device=dev)
        self.cache = lib.PagedCache(kv[0], kv[1])
        self.table = torch.randperm(pages, device=dev, generator=gen).to(torch.int32)[None]     # any pages in any order
        self.lengths = torch.zeros(1, dtype=torch.int32, device=dev)
        self.total = torch.zeros(1, dtype=torch.int32, device=dev)
        self.sequences = lib.Sequences(self.table, self.lengths, pages * PAGE)
        shape = (1, kv_heads, pages * PAGE)
        self.bias, self.weights = torch.zeros(shape, device=dev), torch.zeros(shape, device=dev)
        self.ids = torch.full(shape, -1, dtype=torch.int32, device=dev)
        need = max(lib.sttm_paged_attention_workspace_bytes(self.cache, self.sequences, q_heads, True),
                   lib.sttm_cache_evict_workspace_bytes(self.cache, self.sequences))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)

    def append(self, rows, positions):
        """Rows' keys and values behind what is cached; their queries [n, q_heads, HEAD_DIM]."""
        n, kv = rows.shape[0], self.kv_heads
        qkv = (rows @ self.weight).view(n, -1, HEAD_DIM)
        slot = self.lengths.long() + torch.arange(n, device=rows.device)
        slots = self.table[0].long()[slot // PAGE] * PAGE + slot % PAGE
        q = torch.empty(n, self.q_heads, HEAD_DIM, dtype=rows.dtype, device=rows.device)
        self.ctx.sttm_qk_norm_rope(qkv[:, :-2 * kv], qkv[:, -2 * kv:-kv], qkv[:, -kv:], q, cache=self.cache, slots=slots,
                                   q_weight=self.q_norm, k_weight=self.k_norm, rope=lib.Rope(positions, self.inv_freq))
        self.lengths += n
        self.total += n
        return q

    def attend(self, q):
        """One new token's attention over the cache; every key's weight is added up."""
        out = torch.empty_like(q)
        self.ctx.sttm_paged_attention(q, self.cache, self.sequences, out, HEAD_DIM ** -0.5, key_bias=self.bias, weights_in=self.weights,
                                      weights_out=self.weights, workspace=self.workspace)
        return out

    def evict(self, keep, sink, recent):
        self.ctx.sttm_cache_evict(self.cache, self.sequences, keep, self.lengths, self.weights, self.weights, self.ids, self.ids,
                                  total=self.total, sink=sink, recent=recent, bias_in=self.bias, bias_out=self.bias, workspace=self.workspace)


def run(cfg, keep=0.5, steps=32, cache_keep=0.5):
    dev = torch.device("cuda:0")
    ctx = lib.Sttm(0)
    feats = torch.from_numpy(wl.generate(cfg).view("int16")).to(dev).view(torch.bfloat16)
    rows, counts, index = merge(ctx, feats, keep)
    n, width = rows.shape
    q_heads, kv_heads = max(1, width // HEAD_DIM), max(1, width // HEAD_DIM // 7)
    q_heads = q_heads // kv_heads * kv_heads
    layer = Layer(ctx, width, q_heads, kv_heads, n + 2 * steps, dev)
    layer.append(rows, index)
    layer.bias[:, :, :n] = counts.float().log()
    gen = torch.Generator(device=dev).manual_seed(1)
    outs = []

    def answer(count):
        for _ in range(count):
            token = torch.randn(1, width, device=dev, generator=gen).to(torch.bfloat16)
            outs.append(layer.attend(layer.append(token, layer.total.clone())))

    answer(steps)
    before = layer.attend(q := torch.randn(1, q_heads, HEAD_DIM, device=dev, generator=gen).to(torch.bfloat16))
    full = int(layer.lengths)
    layer.evict((layer.lengths * cache_keep).to(torch.int32), sink=4, recent=steps)
    after = layer.attend(q)
    answer(steps)
    torch.cuda.synchronize()
    return {"video_tokens": feats[..., 0].numel(), "kept": n, "cached": full, "cached_after": int(layer.lengths), "steps": len(outs),
            "similarity": float(torch.cosine_similarity(before.float().flatten(), after.float().flatten(), 0)),
            "finite": bool(torch.isfinite(torch.cat(outs).float()).all())}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--frames", type=int, default=64)
    p.add_argument("--keep", type=float, default=0.5)
    p.add_argument("--steps", type=int, default=32)
    p.add_argument("--cache-keep", type=float, default=0.5)
    a = p.parse_args()
    print(run(wl.small_variant(wl.CONFIGS[1], T=a.frames), a.keep, a.steps, a.cache_keep))
