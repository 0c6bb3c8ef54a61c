"""lsa_chunk_attn where a workgroup's keys need more page-table entries than it stages at a time (31 tiles with pages of one token, 95 of
three, 511 of 16, 2046 of 64); lsa_prefill_attn with rows as far apart as they may be; and the same sequence in a call whose keys are cut into pieces
and in one that leaves them whole. Tolerances: tests/prompt_check.py."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.prompt_check import BF16, DEV, cached, check_chunks, check_prompts, chunks, compare, i32, offsets, prompts, run_chunks, run_prompts, sees

pytestmark = pytest.mark.gpu


def C(H, nk, d=128, fp8=False, k_sink=0, k_swa=0):
    return lsa.DecodeAttnParams(H, nk, d, d, False, d ** -0.5, fp8, k_sink, k_swa)


def _whole(prm, x):
    """Nothing is cut: a workgroup walks all keys of its rows."""
    assert lsa.chunk_attn_workspace_size(prm, len(x["new"]), sum(x["new"]), x["table"].shape[1], x["page"]) == 0
    return run_chunks(prm, x)


def _check_tokens(prm, x, out, lse, b, tokens):
    """The rows of some tokens of sequence b against 64 bits."""
    n, c, group = x["new"][b], x["ctx_list"][b], prm.n_heads // prm.n_kv_heads
    k, mapped = cached(x, "k", b, c, prm.fp8)
    v, _ = cached(x, "v", b, c, prm.fp8)
    tokens = torch.tensor(tokens, device=DEV)
    seen, at = sees(n, c, True, prm.k_sink, prm.k_swa, mapped)[tokens], x["at"][b] + tokens
    for head in range(prm.n_kv_heads):
        hs = slice(head * group, (head + 1) * group)
        compare(out[at, hs], lse[at, hs], x["q"][at, hs].double(), k[head], v[head], seen, prm.sm_scale, (b, n, c, head), extra=2 if prm.fp8 else 0)


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (64, True), (128, True)])
@pytest.mark.parametrize("page", [1, 3])
@pytest.mark.parametrize("sink,swa", [(0, 0), (2100, 2500)], ids=["all", "window"])
@pytest.mark.parametrize("holes", [(), (2500, 2501, 2900)], ids=["mapped", "holes"])
def test_more_pages_than_are_staged(d, fp8, page, sink, swa, holes):
    """9000 positions: five stretches of 1984 with pages of one token, two of 6080 with pages of three. Unmapped pages in one stretch alone; a sink and a
    window that each take two stretches."""
    prm = C(96, 2, d, fp8, sink, swa)
    x = chunks(prm, [1400, 3], [9000, 2100], page, seed=page, bad=[(0, p) for p in holes])
    out, lse = _whole(prm, x)
    check_chunks(prm, x, out, lse)


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (64, True), (128, True)])
@pytest.mark.parametrize("sink,swa", [(0, 0), (7000, 8000)], ids=["all", "window"])
def test_pieces_of_more_pages_than_are_staged(d, fp8, sink, swa):
    """Pieces of about 48 tiles, where 31 are a stretch with pages of one token; unmapped pages."""
    prm = C(16, 16, d, fp8, sink, swa)
    x = chunks(prm, [300, 5], [20000, 9000], 1, seed=d, bad=[(0, 2500), (0, 19000), (1, 8000)])
    assert lsa.chunk_attn_workspace_size(prm, 2, 305, 20000, 1) > 0
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (64, True), (128, True)])
@pytest.mark.parametrize("page,ctx", [(16, 33000), (64, 131100), (100, 204700)])
@pytest.mark.parametrize("where", [None, "first", "last"])
def test_long_tables(d, fp8, page, ctx, where):
    """A second stretch of a few tiles behind one of 2046 pages: whole tiles of a page, pages that are less than a tile and pages that end inside one; an
    unmapped page in neither, in the first or in the last stretch."""
    prm = C(128, 1, d, fp8)
    x = chunks(prm, [1100], [ctx], page, seed=page, bad=[] if where is None else [(0, 700 if where == "first" else ctx // page - 1)])
    assert x["table"].shape[1] > 2046
    out, lse = _whole(prm, x)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    _check_tokens(prm, x, out, lse, 0, [0, 1, 63, 500, 1098, 1099])


@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("lens", [[70, 1, 130, 64], [600]], ids=["whole", "cut"])
@pytest.mark.parametrize("odd", [False, True])
def test_rows_far_apart(d, lens, odd):
    """Tokens 2^24 - 8 elements apart, the most that is taken (a tile's last row lies 2.11e9 bytes behind its first): the bits of the contiguous
    call; `odd`: with a value that is no number, whose rows are computed on another path."""
    prm = lsa.PrefillAttnParams(6, 2, d, min(d, 128), d ** -0.5)
    x = prompts(prm, lens, lens, seed=d, fused=True)
    n, a, b = sum(lens), 6 * d, 8 * d
    assert (lsa.prefill_attn_workspace_size(prm, len(lens), n, n) > 0) == (len(lens) == 1)
    if odd:
        x["v"][50, 1, 3] = float("nan")
    near = {name: x[name].contiguous() for name in "qkv"}
    want = run_prompts(prm, dict(x, **near))
    if not odd:
        check_prompts(prm, dict(x, **near), *want)
    width = b + 2 * prm.d_v
    far = torch.empty((n - 1) * (2 ** 24 - 8) + width, dtype=BF16, device=DEV).as_strided((n, width), (2 ** 24 - 8, 1))
    for name, lo, hi in (("q", 0, a), ("k", a, b), ("v", b, width)):
        far[:, lo:hi].copy_(near[name].flatten(1))
    y = dict(x, q=far[:, :a].unflatten(1, (6, d)), k=far[:, a:b].unflatten(1, (2, d)), v=far[:, b:].unflatten(1, (2, prm.d_v)))
    got = run_prompts(prm, y)
    assert y["k"].stride(0) == 2 ** 24 - 8 and torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[1], want[1])


def _agree(a, b, v):
    """Two calls' (out, lse) of the same rows. With at most 64 for scale sum |q_i k_i| (|q| |k| scale of these inputs is below 50), 192 wide, and 3000 keys,
    e <= 194 * 2^-23 * 64 = 2^-9.4: an output is within (2 * 2^-8 (1 + 2^-8) + 2 e + 3000 * 2^-23 + 2^-18) < 3 * 2^-8 of what the largest |v| bounds,
    an lse, which is below 15, within e + 3000 * 2^-23 + 2^-14 < 2^-9."""
    assert float((a[0].float() - b[0].float()).abs().max()) <= 2 * 3 * 2.0 ** -8 * float(v.abs().max())
    assert float((a[1] - b[1]).abs().max()) <= 2 * 2.0 ** -9


@pytest.mark.parametrize("fp8", [False, True])
def test_a_sequence_of_a_whole_call_in_a_cut_one(fp8):
    """The last sequence of a call that is too large to be cut, alone on the same pages, where it is cut."""
    prm = C(32, 8, 128, fp8)
    new, ctx = [1500] * 4 + [1], [2500, 1500, 1600, 1555, 3000]
    x = chunks(prm, new, ctx, 64, seed=9)
    whole = _whole(prm, x)
    y = dict(x, q=x["q"][6000:].contiguous(), cu=i32([0, 1]), ctx=i32([3000]), table=x["table"][4:].contiguous(), new=[1], ctx_list=[3000], at=[0, 1])
    assert lsa.chunk_attn_workspace_size(prm, 1, 1, y["table"].shape[1], 64) > 0
    cut = run_chunks(prm, y)
    check_chunks(prm, x, *whole)
    check_chunks(prm, y, *cut)
    _agree((whole[0][6000:], whole[1][6000:]), cut, cached(y, "v", 0, 3000, fp8)[0])


@pytest.mark.parametrize("d", [64, 128, 192])
def test_a_prompt_of_a_whole_call_in_a_cut_one(d):
    """The last parts of prompts, packed with others and alone."""
    prm = lsa.PrefillAttnParams(32, 8, d, min(d, 128), d ** -0.5)
    n_q, n_k = [1500] * 3 + [20], [1500, 1700, 1500, 2500]
    x = prompts(prm, n_q, n_k, seed=d)
    assert lsa.prefill_attn_workspace_size(prm, 4, sum(n_q), sum(n_k)) == 0
    whole = run_prompts(prm, x)
    y = dict(x, q=x["q"][4500:], k=x["k"][4700:], v=x["v"][4700:], cu_q=i32([0, 20]), cu_kv=i32([0, 2500]), n_q=[20], n_k=[2500], at=offsets([20]),
             kv_at=offsets([2500]))
    assert lsa.prefill_attn_workspace_size(prm, 1, 20, 2500) > 0
    cut = run_prompts(prm, y)
    check_prompts(prm, x, *whole)
    check_prompts(prm, y, *cut)
    _agree((whole[0][4500:], whole[1][4500:]), cut, y["v"])


@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("n,c,top", [(130, 130, 70), (16, 5000, 4000), (16, 5000, 20)], ids=["whole", "cut", "cut, before"])
def test_an_infinite_value_of_no_weight(d, n, c, top):
    """One key whose score is hundreds above all others: its value is the output, but for the dimensions in which a value attended to is not finite."""
    prm = lsa.PrefillAttnParams(2, 1, d, min(d, 128), 0.125)
    assert (lsa.prefill_attn_workspace_size(prm, 1, n, c) > 0) == (c == 5000)
    x = prompts(prm, [n], [c], seed=d)
    x["q"].fill_(8)
    x["k"].zero_()
    x["k"][top] = 8
    x["v"][10, 0, 5], x["v"][30, 0, 6], x["v"][31, 0, 7] = float("inf"), float("-inf"), float("nan")
    out, _ = run_prompts(prm, x)
    rows = out[top + 1:] if c == n else out
    finite = torch.ones(prm.d_v, dtype=torch.bool, device=DEV)
    finite[5:8] = False
    assert not torch.isfinite(rows[..., ~finite]).any()
    assert torch.equal(rows[..., finite], x["v"][top].expand(rows.shape)[..., finite])
