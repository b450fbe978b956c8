"""Several questions about one video whose reduced tokens are stored once: two ways for a language model to look at them.

    python examples/questions_about_one_video.py [--frames 64] [--keep 0.5] [--steps 16]

The layers' weights and the questions' tokens are random: this shows the calls in their order, not a model.

  1. merge: the video's tokens to a budget, with counts and position indices
  2. a layer of its own that looks at the video: sttm_cross_attention of the questions' tokens to keys and values of the reduced
     rows, as sttm_reduce packs them, then sttm_residual_norm with a gate adds the result and norms the sum for the next block
  3. a layer that has the video in front of every question: its keys and values once, in pages of a cache that all questions share as their
     prefix, each question's own tokens in pages of its own; sttm_shared_attention over both, for all of a question's tokens at once and
     then for one token of every answer a step
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from answer_from_reduced_video import HEAD_DIM, PAGE, lib, merge, wl  # noqa: E402


class VideoLayer:
    """Cross-attention to the video's rows, gated."""

    def __init__(self, ctx, rows, counts, heads, kv_heads, gen):
        width, dev = rows.shape[1], rows.device
        self.ctx, self.heads = ctx, heads
        self.to_q, self.to_kv, self.to_out = (_weight(a, b, gen) for a, b in ((width, heads * HEAD_DIM), (width, 2 * kv_heads * HEAD_DIM), (heads * HEAD_DIM, width)))
        kv = (rows @ self.to_kv).view(-1, 2 * kv_heads, HEAD_DIM)            # once: no token of an answer changes them
        self.kv, self.bias, self.n = kv, counts.float().log(), rows.shape[0]
        self.gate = torch.full((1, 1), 0.3, dtype=rows.dtype, device=dev)
        self.norm = lib.Norm(lib.STTM_NORM_RMS, torch.ones(width, dtype=rows.dtype, device=dev))

    def __call__(self, x, h):
        """x + tanh(gate) * norm(what the tokens see), and its norm."""
        q = (h @ self.to_q).view(-1, self.heads, HEAD_DIM)
        kv_heads, out = self.kv.shape[1] // 2, torch.empty_like(q)
        # (all tokens look at the one video: one sequence of states, one of tokens)
        states = lib.States(self.kv[:, :kv_heads], self.kv[:, kv_heads:], torch.tensor([0, self.n], device=x.device))
        workspace = torch.empty(lib.sttm_cross_attention_workspace_bytes(states, len(x), self.heads), dtype=torch.uint8, device=x.device)
        self.ctx.sttm_cross_attention(q, states, out, HEAD_DIM ** -0.5, q_offsets=torch.tensor([0, len(x)], device=x.device), key_bias=self.bias,
                                      workspace=workspace)
        y, r, h = out.flatten(1) @ self.to_out, torch.empty_like(x), torch.empty_like(x)
        self.ctx.sttm_residual_norm(x, y, r, h, post=self.norm, pre=self.norm, gate=self.gate, gate_tanh=True)
        return r, h


class PrefixLayer:
    """Attention with the video in front: the prefix's pages first in the pool, then those of each question."""

    def __init__(self, ctx, rows, counts, positions, slots, heads, kv_heads, gen):
        width, dev = rows.shape[1], rows.device
        self.ctx, self.heads, self.kv_heads = ctx, heads, kv_heads
        self.to_qkv, self.to_out = _weight(width, (heads + 2 * kv_heads) * HEAD_DIM, gen), _weight(heads * HEAD_DIM, width, gen)
        self.inv_freq = 1e6 ** (-torch.arange(HEAD_DIM // 2, device=dev, dtype=torch.float32) / (HEAD_DIM // 2))
        self.norm = lib.Norm(lib.STTM_NORM_RMS, torch.ones(width, dtype=rows.dtype, device=dev))
        n, batch, each = len(rows), len(slots), -(-max(slots) // PAGE)
        of_video = -(-n // PAGE)
        pool = torch.zeros(2, of_video + batch * each, kv_heads, PAGE, HEAD_DIM, dtype=rows.dtype, device=dev)
        self.cache = lib.PagedCache(pool[0], pool[1])
        pages = torch.arange(of_video + batch * each, dtype=torch.int32, device=dev)
        self.table, self.lengths = pages[of_video:].view(batch, each), torch.zeros(batch, dtype=torch.int32, device=dev)
        self.own = lib.Sequences(self.table, self.lengths, each * PAGE)
        self.video = lib.Sequences(pages[:of_video].view(1, -1), torch.tensor([n], dtype=torch.int32, device=dev), n)
        self.groups = torch.tensor([0, batch], dtype=torch.int32, device=dev)
        self.bias = counts.float().log().expand(1, kv_heads, n).contiguous()
        self.last = int(positions.max()) + 1
        self._project(rows, positions, torch.arange(n, device=dev))

    def _project(self, h, positions, slots):
        qkv, kv = (h @ self.to_qkv).view(len(h), -1, HEAD_DIM), self.kv_heads
        q = torch.empty(len(h), self.heads, HEAD_DIM, dtype=h.dtype, device=h.device)
        self.ctx.sttm_qk_norm_rope(qkv[:, :-2 * kv], qkv[:, -2 * kv:-kv], qkv[:, -kv:], q, cache=self.cache, slots=slots,
                                   rope=lib.Rope(positions.to(torch.int32), self.inv_freq))
        return q

    def __call__(self, x, h, tokens):
        """tokens[b] new ones of question b, one question behind the other in x and h."""
        dev = x.device
        new = torch.tensor(tokens, device=dev)
        of = torch.repeat_interleave(torch.arange(len(tokens), device=dev), new)
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), new.cumsum(0)])
        at = self.lengths.long()[of] + torch.arange(len(of), device=dev) - offsets[of]
        q = self._project(h, self.last + at, self.table.long()[of, at // PAGE] * PAGE + at % PAGE)
        self.lengths += new
        out = torch.empty_like(q)
        workspace = torch.empty(lib.sttm_shared_attention_workspace_bytes(self.cache, self.video, self.own, len(of), self.heads), dtype=torch.uint8, device=dev)
        self.ctx.sttm_shared_attention(q, self.cache, self.video, self.groups, self.own, out, HEAD_DIM ** -0.5, q_offsets=offsets, prefix_bias=self.bias,
                                       workspace=workspace)
        y, r, h = out.flatten(1) @ self.to_out, torch.empty_like(x), torch.empty_like(x)
        self.ctx.sttm_residual_norm(x, y, r, h, pre=self.norm)
        return r, h


def _weight(rows, columns, gen):
    return (torch.randn(rows, columns, device=gen.device, generator=gen) / math.sqrt(rows)).to(torch.bfloat16)


def run(cfg, keep=0.5, questions=(12, 30, 7), steps=16):
    dev = torch.device("cuda:0")
    ctx = lib.Sttm(0)
    feats = torch.from_numpy(wl.generate(cfg).view("int16")).to(dev).view(torch.bfloat16)
    rows, counts, index = merge(ctx, feats, keep)
    width = rows.shape[1]
    heads, kv_heads = max(1, width // HEAD_DIM), max(1, width // HEAD_DIM // 7)
    heads = heads // kv_heads * kv_heads
    gen = torch.Generator(device=dev).manual_seed(2)
    looks = VideoLayer(ctx, rows, counts, heads, kv_heads, gen)
    attends = PrefixLayer(ctx, rows, counts, index, [n + steps for n in questions], heads, kv_heads, gen)
    first = lib.Norm(lib.STTM_NORM_RMS, torch.ones(width, dtype=rows.dtype, device=dev))
    finite, answers = True, 0
    for tokens in [list(questions)] + [[1] * len(questions)] * steps:
        x = torch.randn(sum(tokens), width, device=dev, generator=gen).to(torch.bfloat16)
        h = torch.empty_like(x)
        ctx.sttm_residual_norm(x, None, None, h, pre=first)
        x, h = looks(x, h)
        x, h = attends(x, h, tokens)
        finite = finite and bool(torch.isfinite(x.float()).all()) and bool(torch.isfinite(h.float()).all())
        answers += len(tokens) if tokens == [1] * len(questions) else 0
    return {"video_tokens": feats[..., 0].numel(), "kept": len(rows), "cached": attends.lengths.tolist(), "answers": answers, "finite": finite}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--frames", type=int, default=64)
    p.add_argument("--keep", type=float, default=0.5)
    p.add_argument("--steps", type=int, default=16)
    a = p.parse_args()
    print(run(wl.small_variant(wl.CONFIGS[1], T=a.frames), a.keep, steps=a.steps))
