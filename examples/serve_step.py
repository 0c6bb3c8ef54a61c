#!/usr/bin/env python3
"""Serving steps of two layers over paged caches: prompts are appended, then one token per sequence and step.

    python examples/serve_step.py [--batch 4] [--prompt 700] [--steps 8]

The dense layer has 32 query heads on 8 key heads in an fp8 cache; a step is two calls:
  cache_append   rotates queries and keys, writes keys and values to the new tokens' rows
  decode_attn    attends over every cached position
The LSA layer has the MLA latent cache and fp8 indexer keys; a step is five:
  cache_append   (indexer) rotates its queries and keys, quantises the keys, returns the rows written
  block_keys_update   keeps the block cache of those rows current
  cache_append   (latent) writes [latent | rotated part], rotates the absorbed queries
  index_decode   selects positions;   sparse_attn   attends to them
While a context fits the index budget, the LSA layer attends to all of it: its output is then that of
decode_attn over the latent cache, which the script compares. Projections are random numbers of their shapes."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_01662_amd import lsa  # noqa: E402

PAGE = 64
BF16, FP8 = torch.bfloat16, torch.float8_e4m3fn


def rope_table(n_pos: int, dim: int, dev, base: float = 10000.0) -> torch.Tensor:
    """[n_pos, dim] fp32: dim / 2 cosines, then as many sines, of each position."""
    freq = base ** (-torch.arange(dim // 2, dtype=torch.float64, device=dev) / (dim // 2))
    angle = torch.arange(n_pos, dtype=torch.float64, device=dev)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


class Pages:
    """Page table of `batch` sequences of up to `capacity` tokens, their pages dealt in random order."""

    def __init__(self, batch: int, capacity: int, dev, seed: int = 0):
        width = -(-capacity // PAGE)
        g = torch.Generator().manual_seed(seed)
        self.n_phys = batch * width
        self.table = torch.randperm(self.n_phys, generator=g).view(batch, width).to(torch.int32).to(dev)


class DenseLayer:
    H, HKV, D = 32, 8, 128

    def __init__(self, pages: Pages, n_pos: int, dev):
        self.pages, shape = pages, (pages.n_phys, self.HKV, PAGE, self.D)
        self.k, self.v = (torch.zeros(shape, dtype=torch.uint8, device=dev).view(FP8) for _ in range(2))
        self.ks, self.vs = (torch.zeros(shape[:3], device=dev) for _ in range(2))
        self.rope = rope_table(n_pos, self.D, dev)
        self.ap = lsa.AppendParams(self.H, self.HKV, self.D, self.D, rot_dim=self.D, fp8=True)
        self.at = lsa.DecodeAttnParams(self.H, self.HKV, self.D, self.D, False, self.D ** -0.5, fp8=True)

    def append(self, qkv, **where):
        """qkv [n_tok, (H + 2 HKV) D]: one fused projection, taken as slices. Returns the rotated queries."""
        h, k = self.H * self.D, self.HKV * self.D
        q, _ = lsa.cache_append(self.ap, qkv[:, h:h + k].unflatten(1, (self.HKV, self.D)), self.k, rope=self.rope,
                                v=qkv[:, h + k:].unflatten(1, (self.HKV, self.D)), v_cache=self.v, k_scale=self.ks,
                                v_scale=self.vs, q=qkv[:, :h].unflatten(1, (self.H, self.D)),
                                page_table=self.pages.table, **where)
        return q

    def step(self, qkv, ctx):
        q = self.append(qkv, ctx_len=ctx)
        return lsa.decode_attn(self.at, q, self.k, self.v, ctx, page_table=self.pages.table, k_scale=self.ks,
                               v_scale=self.vs)[0]


class LSALayer:
    H, LATENT, ROT, HI, DI = 64, 512, 64, 32, 128

    def __init__(self, pages: Pages, n_pos: int, dev):
        self.pages = pages
        self.kv = torch.zeros((pages.n_phys, PAGE, self.LATENT + self.ROT), dtype=BF16, device=dev)
        self.ik = torch.zeros((pages.n_phys * PAGE, self.DI), dtype=torch.uint8, device=dev)
        self.iks = torch.zeros((pages.n_phys * PAGE,), device=dev)
        self.ip = lsa.IndexParams(self.HI, self.DI, True, PAGE, PAGE, keep_pages=16, k_sparse=768, k_sink=4, k_swa=256,
                                  run_align=PAGE)
        self.block = lsa.block_keys(self.ip, self.ik, self.iks)
        self.rope = rope_table(n_pos, self.ROT, dev)
        self.iap = lsa.AppendParams(self.HI, 1, self.DI, rot_dim=self.ROT, interleaved=True, fp8=True)
        self.ap = lsa.AppendParams(self.H, 1, self.LATENT + self.ROT, rot_start=self.LATENT, rot_dim=self.ROT,
                                   interleaved=True)
        self.attn = lsa.AttnParams(sm_scale=192 ** -0.5, **lsa.MLA)
        self.dense = lsa.DecodeAttnParams(self.H, 1, 576, 512, True, 192 ** -0.5)

    def append(self, x, **where):
        """x: the layer's projections (see projections). Returns the rotated indexer and absorbed queries."""
        qi, rows = lsa.cache_append(self.iap, x["ik"], self.ik.view(-1, PAGE, self.DI), k_scale=self.iks.view(-1, PAGE),
                                    rope=self.rope, q=x["iq"], rows=True, page_table=self.pages.table, **where)
        lsa.block_keys_update(self.ip, rows, self.ik, self.iks, self.block)
        q, _ = lsa.cache_append(self.ap, x["c"], self.kv, k_rot=x["k_rot"], q=x["q"], q_rot=x["q_rot"], rope=self.rope,
                                page_table=self.pages.table, **where)
        return qi, q

    def step(self, x, ctx):
        qi, q = self.append(x, ctx_len=ctx)
        sel = lsa.index_decode(self.ip, ctx, self.pages.table, PAGE, self.pages.n_phys, qi, x["w"], self.ik, self.iks,
                               self.block, runs=False)
        out, _ = lsa.sparse_attn(self.attn, q, self.kv, None, sel["idx"], sel["count"], page_table=self.pages.table,
                                 kv_page_size=PAGE)
        return out, q

    def dense_step(self, q, ctx):
        """The same attention over the whole context."""
        return lsa.decode_attn(self.dense, q, self.kv, None, ctx, page_table=self.pages.table)[0]


def projections(n: int, g) -> tuple[torch.Tensor, dict]:
    """Random projections of n tokens: the dense layer's fused qkv, and the LSA layer's."""
    def r(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=g.device).mul_(scale).to(BF16)
    d, l = DenseLayer, LSALayer
    qkv = r(n, (d.H + 2 * d.HKV) * d.D)
    x = dict(iq=r(n, l.HI, l.DI, scale=l.DI ** -0.5), ik=r(n, 1, l.DI, scale=l.DI ** -0.5), q=r(n, l.H, l.LATENT),
             q_rot=r(n, l.H, l.ROT), c=r(n, 1, l.LATENT), k_rot=r(n, 1, l.ROT),
             w=torch.rand((n, l.HI), generator=g, device=g.device))
    return qkv, x


def run(batch: int, prompt: int, steps: int, dev=torch.device("cuda:0"), seed: int = 0):
    """Appends prompts of up to `prompt` tokens and takes `steps` steps. Returns, per step, (context lengths, dense
    layer's output, LSA layer's output, latent attention over the whole context)."""
    g = torch.Generator(device=dev).manual_seed(seed)
    ctx = torch.randint(1, prompt + 1, (batch,), generator=g, device=dev).to(torch.int32)
    pages = Pages(batch, prompt + steps, dev, seed)
    dense, sparse = DenseLayer(pages, prompt + steps, dev), LSALayer(pages, prompt + steps, dev)
    # the prompts' tokens, all sequences in one call each
    seq = torch.repeat_interleave(torch.arange(batch, device=dev), ctx.long())
    pos = torch.arange(seq.numel(), device=dev) - (ctx.long().cumsum(0) - ctx.long())[seq]
    where = dict(seq=seq.to(torch.int32), pos=pos.to(torch.int32))
    qkv, x = projections(seq.numel(), g)
    dense.append(qkv, **where)
    sparse.append(x, **where)
    outs = []
    for _ in range(steps):
        ctx = ctx + 1
        qkv, x = projections(batch, g)
        a = dense.step(qkv, ctx)
        b, q = sparse.step(x, ctx)
        outs.append((ctx, a, b, sparse.dense_step(q, ctx)))
    return outs


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--steps", type=int, default=8)
    args = ap.parse_args()
    outs = run(args.batch, args.prompt, args.steps)
    budget = 4 + 256 + 768
    for i, (ctx, a, b, c) in enumerate(outs):
        whole = ctx <= budget          # every position of these contexts is in the index list
        diff = (b.float() - c.float()).abs().amax((1, 2))[whole]
        print(f"step {i}: contexts {ctx.tolist()}, dense |o| {a.float().abs().mean():.4f}, LSA against the whole context: "
              f"{diff.max().item() if diff.numel() else float('nan'):.1e} (of {int(whole.sum())} within the index budget)")


if __name__ == "__main__":
    main()
