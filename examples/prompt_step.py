#!/usr/bin/env python3
"""Prompts of two layers over paged caches, whole and in chunks beside the single tokens of other sequences.

    python examples/prompt_step.py [--batch 4] [--prompt 700] [--chunk 256] [--steps 8]

The grouped layer (32 query heads on 8 key heads of 128, queries and keys normed per head, fp8 or bf16 cache):
  norm_append    norms and rotates queries and keys, writes keys and values to the new tokens' rows; keeps the keys of a whole prompt
  prefill_attn   a whole prompt attends to its own keys and values, packed with others
  chunk_attn     chunks of prompts, and single tokens, attend to what the cache holds
The latent layer (64 heads, the MLA latent cache):
  norm_append    norms the latent, rotates its position part, writes [latent | position part]
  cache_read     reads the rows of a prompt's earlier chunks back, for their up-projection to keys and values of every head
  prefill_attn   the chunk's queries attend to them, 192 / 128 wide
Projections are random numbers of their shapes."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from examples.serve_step import BF16, FP8, PAGE, Pages, rope_table  # noqa: E402
from paper_2608_01662_amd import lsa  # noqa: E402


def offsets(lens, dev):
    return torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device=dev)


def places(new, ctx, dev):
    """Sequence and position of every one of the new[b] last tokens of ctx[b]."""
    seq = [b for b, n in enumerate(new) for _ in range(n)]
    pos = [c - n + i for n, c in zip(new, ctx) for i in range(n)]
    return dict(seq=torch.tensor(seq, dtype=torch.int32, device=dev), pos=torch.tensor(pos, dtype=torch.int32, device=dev))


class GroupedLayer:
    H, HKV, D = 32, 8, 128

    def __init__(self, pages: Pages, n_pos: int, dev, fp8: bool = False):
        self.pages, shape = pages, (pages.n_phys, self.HKV, PAGE, self.D)
        self.k, self.v = ((torch.zeros(shape, dtype=torch.uint8, device=dev).view(FP8) if fp8 else torch.zeros(shape, dtype=BF16, device=dev))
                          for _ in range(2))
        self.scales = {n: torch.zeros(shape[:3], device=dev) for n in ("k_scale", "v_scale")} if fp8 else {}
        self.rope = rope_table(n_pos, self.D, dev)
        g = torch.Generator(device=dev).manual_seed(1)
        self.wq, self.wk = ((1 + 0.1 * torch.randn(self.D, generator=g, device=dev)).to(BF16) for _ in range(2))
        self.ap = lsa.AppendParams(self.H, self.HKV, self.D, self.D, rot_dim=self.D, fp8=fp8)
        self.prefill = lsa.PrefillAttnParams(self.H, self.HKV, self.D, self.D, self.D ** -0.5)
        self.cached = lsa.DecodeAttnParams(self.H, self.HKV, self.D, self.D, False, self.D ** -0.5, fp8=fp8)

    def heads(self, qkv):
        """q, k, v of a fused projection [n_tok, (H + 2 HKV) D], as slices of it."""
        a, b = self.H * self.D, (self.H + self.HKV) * self.D
        return qkv[:, :a].unflatten(1, (self.H, self.D)), qkv[:, a:b].unflatten(1, (self.HKV, self.D)), qkv[:, b:].unflatten(1, (self.HKV, self.D))

    def append(self, qkv, keys=False, **where):
        """Returns the queries (and, if asked for, the keys) as normed and rotated."""
        q, k, v = self.heads(qkv)
        q, k, _ = lsa.norm_append(self.ap, k, self.k, q_weight=self.wq, k_weight=self.wk, k_out=keys, rope=self.rope, v=v, v_cache=self.v, q=q,
                                  page_table=self.pages.table, **self.scales, **where)
        return q, k

    def prompts(self, qkv, lens):
        """Whole prompts, packed: attention over their own keys and values."""
        q, k = self.append(qkv, keys=True, **places(lens, lens, qkv.device))
        return lsa.prefill_attn(self.prefill, q, k, self.heads(qkv)[2], offsets(lens, qkv.device))

    def chunks(self, qkv, new, ctx):
        """The new[b] last of ctx[b] tokens of every sequence: attention over the cache."""
        q, _ = self.append(qkv, **places(new, ctx, qkv.device))
        return lsa.chunk_attn(self.cached, q, self.k, self.v, offsets(new, qkv.device), torch.tensor(ctx, dtype=torch.int32, device=qkv.device),
                              page_table=self.pages.table, **self.scales)


class LatentLayer:
    H, LATENT, ROT, NOPE, DV = 64, 512, 64, 128, 128

    def __init__(self, pages: Pages, n_pos: int, dev):
        self.pages = pages
        self.kv = torch.zeros((pages.n_phys, PAGE, self.LATENT + self.ROT), dtype=BF16, device=dev)
        g = torch.Generator(device=dev).manual_seed(2)
        self.up = (torch.randn((self.LATENT, self.H * (self.NOPE + self.DV)), generator=g, device=dev) * self.LATENT ** -0.5).to(BF16)
        self.weight = (1 + 0.1 * torch.randn(self.LATENT, generator=g, device=dev)).to(BF16)
        self.rope = rope_table(n_pos, self.ROT, dev)
        d = self.NOPE + self.ROT
        self.ap = lsa.AppendParams(0, 1, self.LATENT + self.ROT, rot_start=self.LATENT, rot_dim=self.ROT, interleaved=True)
        self.read = lsa.CacheReadParams(1, self.LATENT + self.ROT)
        self.prefill = lsa.PrefillAttnParams(self.H, self.H, d, self.DV, d ** -0.5)

    def turned(self, q, pos):
        """Queries with the pairs of their last 64 dims rotated."""
        angle = self.rope[pos.long()][:, None]
        cos, sin = angle[..., :self.ROT // 2], angle[..., self.ROT // 2:]
        a, b = q[..., self.NOPE::2].float(), q[..., self.NOPE + 1::2].float()
        return torch.cat([q[..., :self.NOPE], torch.stack([a * cos - b * sin, a * sin + b * cos], 3).flatten(2).to(BF16)], 2)

    def chunks(self, x, new, ctx):
        """x: q [n_tok, H, 192], c [n_tok, 1, 512], k_rot [n_tok, 1, 64]. The new[b] last of ctx[b] tokens attend to their whole contexts.
        Returns (out, lse), and the queries, keys and values that they come from."""
        dev = x["q"].device
        where, cu = places(new, ctx, dev), offsets(ctx, dev)
        lsa.norm_append(self.ap, x["c"], self.kv, k_weight=self.weight, k_rot=x["k_rot"], rope=self.rope, page_table=self.pages.table, **where)
        rows, _ = lsa.cache_read(self.read, self.kv, cu, sum(ctx), page_table=self.pages.table)
        up = (rows[:, 0, :self.LATENT] @ self.up).unflatten(1, (self.H, self.NOPE + self.DV))
        k = torch.cat([up[..., :self.NOPE], rows[:, :, self.LATENT:].expand(-1, self.H, -1)], 2)
        q, v = self.turned(x["q"], where["pos"]), up[..., self.NOPE:].contiguous()
        return lsa.prefill_attn(self.prefill, q, k, v, offsets(new, dev), cu), (q, k, v)


def projections(n: int, g) -> tuple[torch.Tensor, dict]:
    """Random projections of n tokens: the grouped layer's fused qkv, and the latent layer's."""
    def r(*shape):
        return torch.randn(shape, generator=g, device=g.device).to(BF16)
    d, l = GroupedLayer, LatentLayer
    return r(n, (d.H + 2 * d.HKV) * d.D), dict(q=r(n, l.H, l.NOPE + l.ROT), c=r(n, 1, l.LATENT), k_rot=r(n, 1, l.ROT))


def run(batch: int, prompt: int, chunk: int, steps: int, dev=torch.device("cuda:0"), seed: int = 0, fp8: bool = False):
    """Prompts of up to `prompt` tokens once whole and once in chunks of up to `chunk`, then `steps` single tokens of every sequence.
    Returns (lengths, the whole prompts' outputs, the chunked ones', the latent layer's, per step the outputs of the chunks' operator and
    of the decode operator)."""
    g = torch.Generator(device=dev).manual_seed(seed)
    lens = torch.randint(1, prompt + 1, (batch,), generator=g, device=dev).tolist()
    pages = Pages(batch, prompt + steps, dev, seed)
    whole, layer = (GroupedLayer(pages, prompt + steps, dev, fp8) for _ in range(2))
    latent = LatentLayer(pages, prompt + steps, dev)
    qkv, x = projections(sum(lens), g)
    first = offsets(lens, dev).tolist()
    a, _ = whole.prompts(qkv, lens)
    b = torch.empty_like(a)
    done, parts = [0] * batch, []
    while done != lens:     # sequences of other lengths drop out as they are done
        new = [min(chunk, n - d) for n, d in zip(lens, done)]
        ctx = [d + n for d, n in zip(done, new)]
        at = torch.cat([torch.arange(f + d, f + c, device=dev) for f, d, c in zip(first, done, ctx)])
        b[at] = layer.chunks(qkv[at], new, ctx)[0]
        parts.append((at, latent.chunks({n: t[at] for n, t in x.items()}, new, ctx)[0][0]))
        done = ctx
    c = torch.empty((sum(lens), latent.H, latent.DV), dtype=BF16, device=dev)
    for at, out in parts:
        c[at] = out
    outs, ctx = [], lens
    for _ in range(steps):
        ctx = [n + 1 for n in ctx]
        qkv, _ = projections(batch, g)
        one, _ = layer.chunks(qkv, [1] * batch, ctx)
        length = torch.tensor(ctx, dtype=torch.int32, device=dev)
        q, _ = layer.append(qkv, ctx_len=length)    # (again: the same rows, the same values)
        outs.append((one, lsa.decode_attn(layer.cached, q, layer.k, layer.v, length, page_table=pages.table, **layer.scales)[0]))
    return lens, a, b, c, outs


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--chunk", type=int, default=256)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--fp8", action="store_true")
    args = ap.parse_args()
    lens, a, b, c, outs = run(args.batch, args.prompt, args.chunk, args.steps, fp8=args.fp8)
    print(f"prompts of {lens}: whole against chunks {(a.float() - b.float()).abs().max():.1e} (|o| {a.float().abs().mean():.4f}), "
          f"latent |o| {c.float().abs().mean():.4f}")
    for i, (one, dec) in enumerate(outs):
        print(f"step {i}: single tokens as chunks against decode attention {(one.float() - dec.float()).abs().max():.1e}")


if __name__ == "__main__":
    main()
