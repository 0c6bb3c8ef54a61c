"""lsa_decode_attn where a workgroup's stretch needs more page-table entries than it stages at a time (63 tiles of grouped heads
and 31 of the latent cache with pages of one token), and with many new tokens: against the float64 oracle, with the
tolerances of test_gpu_decode_attn."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_gpu_decode_attn import GQA, MLA, _batch, _check, _params, _run

pytestmark = pytest.mark.gpu


def _holes(x, ctx, first, every):
    """Unmaps pages of a table with pages of one token: every `every`-th position from `first` on, and the first one."""
    for b, c in enumerate(ctx):
        x["table"][b, first:c:every] = -1
        if c > 100:
            x["table"][b, 0] = -1


@pytest.mark.parametrize("sink,swa", [(0, 0), (1300, 690), (150, 1850)], ids=["all", "sink", "window"])
@pytest.mark.parametrize("form,R", [((GQA, 12, 12, 64, False), 1), ((GQA, 24, 12, 128, True), 2)], ids=str)
def test_grouped_heads_whole(form, R, sink, swa):
    """64 tiles in a workgroup, two passes; with a window, tiles of the sink and of the window in one of them."""
    prm = _params(*form, k_sink=sink, k_swa=swa)
    ctx = [2048, 2047, 1, 0, 2020, 1999, 2017, 33, 500] if not swa else [2918, 2048, 1, 0, 2020, 1999, 3500, 33, 500]
    x = _batch(prm, ctx, R, 1, seed=31 + R)
    _holes(x, ctx, 2011, 7)
    assert x["table"].shape[1] > 63 * 32 and lsa.decode_attn_workspace_size(prm, len(ctx), R, x["table"].shape[1], 1) == 0
    out, lse = _run(prm, x)
    _check(prm, x, out, lse)


@pytest.mark.parametrize("sink,swa", [(0, 0), (2600, 2500), (100, 6000)], ids=["all", "sink", "window"])
@pytest.mark.parametrize("form,R", [((GQA, 64, 64, 64, False), 1), ((GQA, 64, 64, 64, True), 3)], ids=str)
def test_grouped_heads_cut(form, R, sink, swa):
    """64 key heads leave eight stretches: of 64 tiles and more each."""
    prm = _params(*form, k_sink=sink, k_swa=swa)
    ctx = [4001, 8100, 33, 6010, 7003]
    x = _batch(prm, ctx, R, 1, seed=41 + R)
    _holes(x, ctx, 2100, 11)
    assert lsa.decode_attn_workspace_size(prm, len(ctx), R, x["table"].shape[1], 1) > 0
    out, lse = _run(prm, x)
    _check(prm, x, out, lse)


@pytest.mark.parametrize("sink,swa", [(0, 0), (1100, 300), (100, 1300)], ids=["all", "sink", "window"])
@pytest.mark.parametrize("heads,R", [(16, 1), (64, 1), (20, 3)])
def test_latent_whole(heads, R, sink, swa):
    """Blocks of 32 and of 64 query rows, up to 48 tiles in a workgroup: two passes of 31."""
    prm = _params(MLA, heads, 1, 576, k_sink=sink, k_swa=swa)
    g = torch.Generator().manual_seed(3)
    ctx = [int(c) for c in torch.randint(0, 200, (160,), generator=g)]
    ctx[0], ctx[7], ctx[40], ctx[159] = 1500, 1024, 993, 1441
    if swa:
        ctx[0], ctx[159] = 3001, 2200
    x = _batch(prm, ctx, R, 1, seed=heads)
    _holes(x, ctx, 1003, 13)
    assert x["table"].shape[1] > 31 * 32 and lsa.decode_attn_workspace_size(prm, len(ctx), R, x["table"].shape[1], 1) == 0
    out, lse = _run(prm, x)
    _check(prm, x, out, lse, rows={b * R + j for b in (0, 1, 7, 39, 40, 100, 159) for j in range(R)})


@pytest.mark.parametrize("sink,swa", [(0, 0), (3500, 2100), (100, 6000)], ids=["all", "sink", "window"])
@pytest.mark.parametrize("heads,R", [(1024, 1), (500, 2)])
def test_latent_cut(heads, R, sink, swa):
    """A thousand query rows of a sequence leave 16 stretches, of more than 31 tiles each."""
    prm = _params(MLA, heads, 1, 576, k_sink=sink, k_swa=swa)
    ctx = [9001, 8000, 8500]
    x = _batch(prm, ctx, R, 1, seed=heads)
    _holes(x, ctx, 1500, 17)
    assert lsa.decode_attn_workspace_size(prm, len(ctx), R, x["table"].shape[1], 1) > 0
    out, lse = _run(prm, x)
    _check(prm, x, out, lse)


@pytest.mark.parametrize("sink,swa", [(0, 0), (4, 300)], ids=["all", "window"])
@pytest.mark.parametrize("form", [(GQA, 32, 8, 128, False), (GQA, 16, 2, 64, True), (GQA, 12, 1, 128, True), (GQA, 5, 5, 64, False), (MLA, 64, 1, 576, False),
                                  (MLA, 16, 1, 576, False), (MLA, 6, 1, 576, False)], ids=str)
@pytest.mark.parametrize("R", [17, 20, 129, 512, 1024])
def test_many_new_tokens(form, R, sink, swa):
    """Chunks of new tokens: as many as 1024 of a sequence, some of them more than it holds; rows at the ends of the
    blocks of query rows and in between, each against its own context. The cache whole and cut."""
    prm = _params(*form, k_sink=sink, k_swa=swa)
    for ctx, width in (([700, 40, 0, R], None), ([2101, R + 1], 70)):
        x = _batch(prm, ctx, R, 64, seed=R, width=max(width or 0, -(-max(ctx) // 64)))
        out, lse = _run(prm, x)
        some = sorted({0, 1, 15, 16, R // 3, R // 2, R - 2, R - 1})
        _check(prm, x, out, lse, rows={b * R + j for b in range(len(ctx)) for j in some})
