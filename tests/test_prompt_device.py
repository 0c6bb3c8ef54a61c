"""The prompt-side operators on tensors of a GPU that is not the current one: they run there, on its stream."""
from __future__ import annotations

import types

import pytest
import torch

from paper_2608_01662_amd import lsa

BF = torch.bfloat16
TWO = pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")


def _calls(dev):
    g = torch.Generator().manual_seed(4)
    x = lambda *s: torch.randn(s, generator=g).to(BF).to(dev)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    k_cache, v_cache = (torch.zeros((48, 2, 64, 64), dtype=BF, device=dev) for _ in range(2))
    table, ctx, cu = torch.arange(48, dtype=torch.int32, device=dev)[None].contiguous(), i32([3000]), i32([0, 3000])
    q, k, rows = lsa.norm_append(lsa.AppendParams(4, 2, 64, 64, 0, 64), x(3000, 2, 64), k_cache, page_table=table, seq=i32([0] * 3000),
                                 pos=torch.arange(3000, dtype=torch.int32, device=dev), v=x(3000, 2, 64), v_cache=v_cache, q=x(3000, 4, 64),
                                 rope=x(3000, 64).float(), q_weight=x(64), k_weight=x(64), k_out=True, rows=True)
    _, v = lsa.cache_read(lsa.CacheReadParams(2, 64, 64), k_cache, cu, 3000, page_table=table, v_cache=v_cache)
    a = lsa.prefill_attn(lsa.PrefillAttnParams(4, 2, 64, 64, 0.125), q, k, v, cu)
    b = lsa.chunk_attn(lsa.DecodeAttnParams(4, 2, 64, 64, False, 0.125), q[-20:], k_cache, v_cache, i32([0, 20]), ctx, page_table=table)
    return [t.cpu() for t in (q, k, rows, v, *a, *b)]


@pytest.mark.gpu
@TWO
@pytest.mark.parametrize("compiled", [True, False])
def test_tensors_of_another_gpu(monkeypatch, compiled):
    want = _calls(torch.device("cuda:0"))
    if not compiled:
        names = ("cache_append", "norm_append", "cache_read", "prefill_attn", "chunk_attn", "decode_attn")
        monkeypatch.setattr(lsa, "_serve", types.SimpleNamespace(**{n: lambda *a: None for n in names}))
    assert torch.cuda.current_device() == 0
    got = _calls(torch.device("cuda:1"))
    assert torch.cuda.current_device() == 0
    for a, b in zip(want, got):
        assert torch.equal(a, b)
