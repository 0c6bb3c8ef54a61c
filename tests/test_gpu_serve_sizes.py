"""lsa_decode_attn calls of more workgroups than one launch of the runtime takes (2^32 threads): rows from all over such a
call against the float64 oracle."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_gpu_decode_attn import GQA, MLA, _check, _params

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16


def _calls_rows(prm, n_seq, R, ctx, width, seqs):
    """A call of n_seq sequences over a few shared pages of 16 tokens, and the rows of some of them against the oracle."""
    g = torch.Generator(device=DEV).manual_seed(5)
    n_phys = 64
    shape = (n_phys, 16, prm.d_qk) if prm.latent else (n_phys, prm.n_kv_heads, 16, prm.d_qk)
    k = torch.randn(shape, generator=g, device=DEV).to(BF)
    v = None if prm.latent else torch.randn(shape, generator=g, device=DEV).to(BF)
    q = torch.empty((n_seq * R, prm.n_heads, prm.d_qk), dtype=BF, device=DEV).normal_(generator=g)
    table = torch.randint(0, n_phys, (n_seq, width), generator=g, device=DEV, dtype=torch.int32)
    out, lse = lsa.decode_attn(prm, q, k, v, ctx, page_table=table, rows_per_seq=R)
    torch.cuda.synchronize()
    for b in seqs:
        rows = slice(b * R, (b + 1) * R)
        some = sorted({0, R // 2, R - 1})
        x = dict(q=q[rows], ctx=ctx[b:b + 1], table=table[b:b + 1], R=R, page=16, k_cache=k)
        if v is not None:
            x["v_cache"] = v
        _check(prm, x, out[rows], lse[rows], rows=set(some))
    return out, lse


@pytest.mark.parametrize("form,n_seq", [((GQA, 64, 64, 64, False), (1 << 18) + 3), ((MLA, 1, 1, 576, False), (1 << 23) + 5)], ids=str)
def test_many_whole_sequences(form, n_seq):
    """One workgroup of 256 (grouped) or 512 threads (latent) per sequence and head."""
    prm = _params(*form)
    ctx = torch.randint(0, 17, (n_seq,), device=DEV, dtype=torch.int32)
    ctx[-1], ctx[n_seq // 2] = 16, 3
    assert lsa.decode_attn_workspace_size(prm, n_seq, 1, 1, 16) == 0
    out, lse = _calls_rows(prm, n_seq, 1, ctx, 1, [0, 1, 777, n_seq // 2, n_seq - 2, n_seq - 1])
    empty = (ctx == 0)
    assert (out[empty] == 0).all() and (lse[empty] == float("-inf")).all() and torch.isfinite(lse[~empty]).all()


def test_many_joined_rows():
    """256 threads of the join per query row, 2^24 and more of them."""
    prm = _params(GQA, 32, 1, 64, False)
    n_seq, R = 8193, 64
    ctx = torch.zeros(n_seq, dtype=torch.int32, device=DEV)
    some = [0, 100, 8191, 8192]
    for b, c in zip(some, (2100, 16, 1500, 2112)):
        ctx[b] = c
    assert lsa.decode_attn_workspace_size(prm, n_seq, R, 132, 16) > 0
    out, lse = _calls_rows(prm, n_seq, R, ctx, 132, some)
    idle = torch.ones(n_seq, dtype=torch.bool, device=DEV)
    idle[some] = False
    assert (out.view(n_seq, R, 32, 64)[idle] == 0).all() and (lse.view(n_seq, R, 32)[idle] == float("-inf")).all()
