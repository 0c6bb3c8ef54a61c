"""The dense layer of examples/serve_step.py over prompts of many pages, step by step, against softmax attention in 64 bits over
what its fp8 cache holds; and calls of no tokens."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests import parity as P
from tests.test_gpu_serve_step import _example

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def test_dense_layer_over_long_prompts():
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(6)
    lens, steps = [1500, 333, 64], 3
    pages = m.Pages(3, max(lens) + steps, DEV)
    layer = m.DenseLayer(pages, max(lens) + steps, DEV)
    ctx = torch.tensor(lens, dtype=torch.int32, device=DEV)
    seq = torch.repeat_interleave(torch.arange(3, device=DEV), ctx.long())
    pos = torch.cat([torch.arange(n, device=DEV) for n in lens])
    layer.append(m.projections(seq.numel(), g)[0], seq=seq.to(torch.int32), pos=pos.to(torch.int32))
    for _ in range(steps):
        ctx = ctx + 1
        qkv, _ = m.projections(3, g)
        out = layer.step(qkv, ctx).double().cpu()
        q = layer.append(qkv, ctx_len=ctx).double().cpu()      # (again: the same rows, the same values)
        for b, n in enumerate(ctx.tolist()):
            at = pages.table[b, :-(-n // m.PAGE)].long()
            k = (layer.k[at].float() * layer.ks[at][..., None]).double().transpose(0, 1).flatten(1, 2)[:, :n].cpu()
            v = (layer.v[at].float() * layer.vs[at][..., None]).double().transpose(0, 1).flatten(1, 2)[:, :n].cpu()
            for h in range(32):
                p = torch.softmax(k[h // 4] @ q[b, h] * layer.at.sm_scale, 0)
                ref = p @ v[h // 4]
                assert float((out[b, h] - ref).abs().max()) <= P.ATOL_O and float((out[b, h] - ref).norm() / ref.norm()) <= P.RTOL_O


def test_calls_of_no_tokens():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    cache = bf(2, 2, 16, 64)
    q, rows = lsa.cache_append(lsa.AppendParams(4, 2, 64, 64, 0, 64), bf(0, 2, 64), cache, page_table=i32(2, 1), pos=i32(0), seq=i32(0), v=bf(0, 2, 64),
                               v_cache=bf(2, 2, 16, 64), q=bf(0, 4, 64), rope=torch.zeros((16, 64), device=DEV), rows=True)
    assert q.shape == (0, 4, 64) and rows.shape == (0,) and cache.count_nonzero() == 0
    out, lse = lsa.decode_attn(lsa.DecodeAttnParams(4, 2, 64, 64, False, 0.125), bf(0, 4, 64), cache, bf(2, 2, 16, 64), i32(0), page_table=i32(0, 1))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
