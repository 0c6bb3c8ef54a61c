"""Numbers that the serving operators' C interface takes in 32 bits are refused where they do not fit, not cut off."""
from __future__ import annotations

from dataclasses import fields, replace

import pytest
import torch

from paper_2608_01662_amd import lsa

APPEND = lsa.AppendParams(4, 2, 64, 64, 0, 64)
ATTN = lsa.DecodeAttnParams(4, 2, 64, 64, False, 0.125, k_sink=4, k_swa=100)


@pytest.mark.parametrize("prm", [APPEND, ATTN], ids=["append", "attention"])
def test_parameters(prm):
    prm.c()
    for f in fields(prm):
        if f.type != "int":
            continue
        for bad in ((1 << 32) + getattr(prm, f.name), 1 << 31, -(1 << 31) - 1):
            with pytest.raises(ValueError, match=f.name):
                replace(prm, **{f.name: bad}).c()


@pytest.mark.gpu
def test_calls():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    ctx = torch.tensor([5, 9], dtype=torch.int32, device="cuda")
    table = torch.arange(2, dtype=torch.int32, device="cuda")[:, None].contiguous()
    attn = lambda prm, **kw: lsa.decode_attn(prm, bf(2, 4, 64), bf(2, 2, 16, 64), bf(2, 2, 16, 64), ctx, page_table=table, **kw)
    attn(ATTN)
    for name in ("k_sink", "k_swa"):
        with pytest.raises(ValueError, match=name):
            attn(replace(ATTN, **{name: (1 << 32) + 7}))
    append = lambda prm, **kw: lsa.cache_append(prm, bf(2, 2, 64), bf(2, 2, 16, 64), page_table=table, v=bf(2, 2, 64), v_cache=bf(2, 2, 16, 64),
                                                q=bf(2, 4, 64), rope=torch.zeros((16, 64), device="cuda"), **kw)
    append(APPEND, ctx_len=ctx)
    with pytest.raises(ValueError, match="rot_start"):
        append(replace(APPEND, rot_start=1 << 32), ctx_len=ctx)
    with pytest.raises(ValueError, match="rows_per_seq"):       # (by position it names no count of tokens)
        append(APPEND, pos=ctx, rows_per_seq=(1 << 32) + 1)
