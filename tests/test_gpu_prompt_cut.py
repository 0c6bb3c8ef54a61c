"""Calls of lsa_prefill_attn and lsa_chunk_attn whose keys are cut into pieces, and calls too large for that, on the same sequences; pieces of
every kind of mask; contexts up to the last position that 31 bits hold. Tolerances: tests/prompt_check.py."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.prompt_check import BF16, DEV, check_chunks, check_prompts, chunks, compare, i32, prompts, run_chunks, run_prompts

pytestmark = pytest.mark.gpu


def C(H, nk, d=128, fp8=False, k_sink=0, k_swa=0):
    return lsa.DecodeAttnParams(H, nk, d, d, False, d ** -0.5, fp8, k_sink, k_swa)


@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("n_q,n_k", [(1, 5000), (40, 9000), (300, 3333), (7, 40000)])
def test_few_rows_of_long_prompts(d, n_q, n_k):
    prm = lsa.PrefillAttnParams(8, 2, d, min(d, 128), d ** -0.5)
    assert lsa.prefill_attn_workspace_size(prm, 3, n_q + 3, n_k + 100) > 0
    x = prompts(prm, [n_q, 3, 0], [n_k, 90, 10], seed=n_q)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("d", [64, 128, 192])
def test_pieces_without_a_mask(d):
    prm = lsa.PrefillAttnParams(4, 4, d, min(d, 128), d ** -0.5, causal=False)
    x = prompts(prm, [5, 300], [7001, 2500], seed=d)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("sink,swa,page", [(0, 3000, 64), (70, 2500, 20), (3000, 100, 64), (100, 4000, 128)])
def test_pieces_of_windows(fp8, sink, swa, page):
    """The sink and the window each in several pieces, pieces that end inside either."""
    prm = C(8, 2, 64, fp8, sink, swa)
    x = chunks(prm, [5, 80, 1], [6000, 5000, 9000], page, seed=swa)
    check_chunks(prm, x, *run_chunks(prm, x))


def test_pieces_without_a_key():
    """Sequences of which every page is unmapped, or all but the last: pieces without a key have no effect."""
    prm = C(16, 2)
    x = chunks(prm, [2, 3, 50], [4000, 4000, 5000], 64, seed=5, bad=[(0, p) for p in range(63)] + [(1, p) for p in range(62)])
    out, lse = run_chunks(prm, x)
    check_chunks(prm, x, out, lse)
    assert (lse[:2] == float("-inf")).all() and torch.isfinite(lse[2:]).all()


@pytest.mark.parametrize("n_seq", [64, 65, 130])
def test_sequences_of_all_sizes(n_seq):
    """Up to 64 sequences are taken largest first, more as they come: every row is written once, whatever the order."""
    g = torch.Generator().manual_seed(n_seq)
    new = torch.randint(0, 12, (n_seq,), generator=g).tolist()
    ctx = [n + int(2 ** (13 * float(torch.rand((), generator=g)))) for n in new]
    prm = C(4, 2, 64, n_seq == 65)
    assert lsa.chunk_attn_workspace_size(prm, n_seq, sum(new), -(-max(ctx) // 64), 64) > 0
    x = chunks(prm, new, ctx, 64, seed=n_seq)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("fp8", [False, True])
def test_calls_too_large_to_be_cut(fp8):
    """More blocks of rows than are cut: each walks its keys alone; and the same sequence in a call that is cut, within both roundings."""
    prm = C(32, 8, 128, fp8)
    new, ctx = [1500] * 4 + [1], [2500, 1500, 1600, 1555, 3000]
    assert lsa.chunk_attn_workspace_size(prm, 5, sum(new), 47, 64) == 0
    x = chunks(prm, new, ctx, 64, seed=9)
    out, lse = run_chunks(prm, x)
    check_chunks(prm, x, out, lse)


def test_heads_over_the_chips_parts():
    """Numbers of key/value heads with every common divisor with 8, more and fewer blocks of rows than turns, too few keys to be cut."""
    for H, nk in ((3, 3), (6, 2), (12, 4), (8, 8), (10, 10), (24, 24), (7, 1)):
        prm = lsa.PrefillAttnParams(H, nk, 64, 64, 0.125)
        n = [190, 0, 1, 260, 60]
        x = prompts(prm, n, n, seed=H)
        assert lsa.prefill_attn_workspace_size(prm, 5, sum(n), sum(n)) == 0
        check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("P,fp8", [(1 << 20, False), ((1 << 20) - 4, False), (1 << 20, True)])
def test_last_positions(P, fp8):
    """Contexts up to the table's end, just below 2^31, whose pages are all one page: the window's and the sink's positions."""
    width = ((1 << 31) - 1) // P
    cap = width * P
    prm = C(4, 1, 64, fp8, 70, 150)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((1, 1, P, 64), generator=g, device=DEV) for _ in range(2))
    scale = {}
    if fp8:
        scale = {"k_scale": torch.rand((1, 1, P), generator=g, device=DEV), "v_scale": torch.rand((1, 1, P), generator=g, device=DEV)}
        k, v = k.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)
    else:
        k, v = k.to(BF16), v.to(BF16)
    table = torch.zeros((2, width), dtype=torch.int32, device=DEV)
    new, ctx = [5, 70], [cap, cap - 1000]
    q = torch.randn((75, 4, 64), generator=g, device=DEV).to(BF16)
    out, lse = lsa.chunk_attn(prm, q, k, v, i32([0, 5, 75]), i32(ctx), page_table=table, **scale)
    at = 0
    for n, c in zip(new, ctx):
        pos = torch.cat([torch.arange(70, device=DEV), torch.arange(c - n - 160, c, device=DEV)])
        rows = [(x[0, 0, pos % P].double() if not fp8 else x.view(torch.uint8)[0, 0, pos % P].view(torch.float8_e4m3fn).double() *
                 scale[s][0, 0, pos % P].double()[:, None]) for x, s in ((k, "k_scale"), (v, "v_scale"))]
        t = torch.arange(c - n, c, device=DEV)[:, None]
        seen = (pos <= t) & ((pos > t - 150) | (pos < 70))
        compare(out[at:at + n], lse[at:at + n], q[at:at + n].double(), *rows, seen, prm.sm_scale, (n, c), extra=2 if fp8 else 0)
        at += n


def test_two_graphs_with_workspaces_of_their_own():
    """Two captured calls, replayed in turn and at once on two streams, give what each gives alone."""
    prm = C(8, 2)
    calls = []      # (with what each graph reads and works in, which has to live as long as it is replayed)
    for seed, new, ctx in ((1, [3, 40], [6000, 4000]), (2, [64], [9000])):
        x = chunks(prm, new, ctx, 64, seed=seed)
        ws = torch.empty(lsa.chunk_attn_workspace_size(prm, len(new), sum(new), x["table"].shape[1], 64), dtype=torch.uint8, device=DEV)
        out, lse = run_chunks(prm, x, workspace=ws)
        want = out.clone(), lse.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lsa.chunk_attn(prm, x["q"], x["k_cache"], x["v_cache"], x["cu"], x["ctx"], page_table=x["table"], out=out, lse=lse, workspace=ws)
        calls.append((graph, out, lse, want, torch.cuda.Stream(), x, ws))
    for _ in range(3):
        for graph, out, lse, _, s, *_ in calls:
            with torch.cuda.stream(s):
                out.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for _, out, lse, want, *_ in calls:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_two_graphs_that_share_a_workspace():
    """Two captured calls of other sizes with one workspace, replayed one after the other, each against its eager result."""
    prm = C(8, 2)
    calls = []
    xs = [chunks(prm, new, ctx, 64, seed=seed) for seed, new, ctx in ((1, [3, 40], [6000, 4000]), (2, [64, 1, 1], [9000, 500, 3000]))]
    ws = torch.empty(max(lsa.chunk_attn_workspace_size(prm, len(x["new"]), sum(x["new"]), x["table"].shape[1], 64) for x in xs), dtype=torch.uint8, device=DEV)
    for x in xs:
        out, lse = run_chunks(prm, x)
        want = out.clone(), lse.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lsa.chunk_attn(prm, x["q"], x["k_cache"], x["v_cache"], x["cu"], x["ctx"], page_table=x["table"], out=out, lse=lse, workspace=ws)
        calls.append((graph, out, lse, want))
    for i in (0, 1, 1, 0, 0, 1):
        graph, out, lse, want = calls[i]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_a_workspace_that_held_something_else():
    """What the workspace holds before a call has no effect."""
    prm = C(8, 2)
    x = chunks(prm, [3, 40], [6000, 4000], 64, seed=3)
    size = lsa.chunk_attn_workspace_size(prm, 2, 43, x["table"].shape[1], 64)
    want = run_chunks(prm, x, workspace=torch.zeros(size, dtype=torch.uint8, device=DEV))
    for fill in (0xFF, 0x7F, 0x01):
        got = run_chunks(prm, x, workspace=torch.full((size,), fill, dtype=torch.uint8, device=DEV))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_offsets_that_do_not_ascend_write_no_row_of_others():
    """Ranges within the tensors that overlap (the offsets are to ascend): whatever is computed, no row outside the ranges is written."""
    prm = C(8, 2)
    x = chunks(prm, [40, 40, 40], [3000, 3000, 3000], 64, seed=4, tail=30)
    x["cu"] = i32([50, 90, 40, 80])
    out, lse = run_chunks(prm, x)
    torch.cuda.synchronize()
    assert (out[:40] == 7.0).all() and (out[90:] == 7.0).all() and (lse[90:] == 7.0).all()
