"""The serving operators on tensors of a GPU that is not the current one: they run there, on its stream."""
from __future__ import annotations

import types

import pytest
import torch

from paper_2608_01662_amd import lsa

BF = torch.bfloat16
TWO = pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")


def _calls(dev):
    """Queries, caches and outputs of an append and an attention of two sequences on `dev`."""
    g = torch.Generator().manual_seed(4)
    x = lambda *s: torch.randn(s, generator=g).to(BF).to(dev)
    k_cache, v_cache = (torch.zeros((2, 2, 16, 64), dtype=BF, device=dev) for _ in range(2))
    ctx = torch.tensor([1, 1], dtype=torch.int32, device=dev)
    table = torch.arange(2, dtype=torch.int32, device=dev)[:, None].contiguous()
    q, rows = lsa.cache_append(lsa.AppendParams(4, 2, 64, 64, 0, 64), x(2, 2, 64), k_cache, page_table=table, ctx_len=ctx, v=x(2, 2, 64),
                               v_cache=v_cache, q=x(2, 4, 64), rope=x(4, 64).float(), rows=True)
    out, lse = lsa.decode_attn(lsa.DecodeAttnParams(4, 2, 64, 64, False, 0.125), q, k_cache, v_cache, ctx, page_table=table)
    return [t.cpu() for t in (q, rows, k_cache, v_cache, out, lse)]


@pytest.mark.gpu
@TWO
@pytest.mark.parametrize("compiled", [True, False])
def test_tensors_of_another_gpu(monkeypatch, compiled):
    want = _calls(torch.device("cuda:0"))
    if not compiled:
        monkeypatch.setattr(lsa, "_serve", types.SimpleNamespace(cache_append=lambda *a: None, decode_attn=lambda *a: None))
    assert torch.cuda.current_device() == 0
    got = _calls(torch.device("cuda:1"))
    assert torch.cuda.current_device() == 0
    for a, b in zip(want, got):
        assert torch.equal(a, b)
