"""lsa_chunk_attn against 64 bits: ragged chunks of new tokens over a paged cache. Tolerances: tests/prompt_check.py."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.prompt_check import BF16, DEV, check_chunks, chunks, i32, run_chunks

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def P(H, nk, d=128, fp8=False, k_sink=0, k_swa=0):
    return lsa.DecodeAttnParams(H, nk, d, d, False, d ** -0.5, fp8, k_sink, k_swa)


FORMS = [(32, 8), (32, 8, 128, True), (16, 1), (4, 4, 64), (4, 4, 64, True), (28, 4, 64, True), (40, 5), (100, 1, 128, True), (1, 1), (96, 2, 64)]
NEW = [1, 0, 2, 31, 64, 1, 65, 130, 0, 7, 300]
CTX = [1, 5, 100, 31, 64, 1000, 127, 129, 0, 513, 700]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("page", [64, 37, 128])
def test_forms_and_lengths(form, page):
    """Every head layout and type; chunks and single tokens side by side, whole prompts, more new tokens than positions (129 of 130)."""
    prm = P(*form)
    x = chunks(prm, NEW, CTX, page, seed=page)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("form", [(32, 8), (8, 8, 64, True), (16, 2, 128, True)], ids=str)
@pytest.mark.parametrize("page", [1, 3, 16, 20, 32, 100, 256, 1000])
def test_page_sizes(form, page):
    prm = P(*form)
    x = chunks(prm, [3, 100, 64, 1], [10, 999, 64, 1500], page, seed=page)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("form", [(8, 2), (3, 3, 64), (16, 2, 128, True)], ids=str)
@pytest.mark.parametrize("sink,swa", [(0, 1), (4, 128), (0, 64), (100, 33), (64, 64), (0, 2000), (700, 100), (1, 65)])
@pytest.mark.parametrize("page", [64, 20])
def test_windows(form, sink, swa, page):
    prm = P(*form, k_sink=sink, k_swa=swa)
    x = chunks(prm, [1, 64, 130, 300, 5, 1], [1, 64, 200, 777, 1500, 900], page, seed=sink + swa)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("form", [(32, 8), (16, 1, 128, True), (8, 8, 64), (28, 4, 64, True)], ids=str)
@pytest.mark.parametrize("page", [64, 48])
def test_long_contexts(form, page):
    """A chunk of 1500 behind 2600, few new tokens of 9001 and single ones."""
    prm = P(*form)
    x = chunks(prm, [1500, 3, 1], [4100, 9001, 6000], page, seed=page)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [64, 16, 100])
def test_pages_without_memory(fp8, page):
    """Unmapped pages (entries of -1, n_phys and -2^31) anywhere, also all of a sequence's: their positions are not attended to."""
    prm = P(8, 2, 128, fp8)
    x = chunks(prm, [70, 1, 33, 5], [700, 400, 200, 90], page, seed=page, bad=[(0, 1), (0, 3), (1, 0), (2, 1)] + [(3, p) for p in range(-(-90 // page))])
    check_chunks(prm, x, *run_chunks(prm, x))


def test_idle_and_impossible_sequences():
    """Lengths of 0, below 0 and beyond the table: rows of zeros; tables wider than any context; rows of no sequence."""
    prm = P(8, 2, 64)
    x = chunks(prm, [3, 70, 1, 2, 0], [40, 100, 9, 64, 33], 16, seed=1, lead=2, tail=3, width=20)
    ctx = [40, -1, 0, 20 * 16 + 1, 33]
    x = dict(x, ctx=i32(ctx), ctx_list=ctx)
    check_chunks(prm, x, *run_chunks(prm, x))


@pytest.mark.parametrize("fp8", [False, True])
def test_what_is_not_attended_to_has_no_effect(fp8):
    """NaN and infinities in cached rows of later tokens and of positions before a window; (fp8: in the scales)."""
    for sink, swa in ((0, 0), (4, 40)):
        prm = P(4, 2, 64, fp8, sink, swa)
        x = chunks(prm, [60, 1], [150, 150], 16, seed=2)
        want = run_chunks(prm, x)
        check_chunks(prm, x, *want)
        for bad in (NAN, INF, -INF) if not fp8 else (NAN, INF):
            y = dict(x)
            names = [n + ("_scale" if fp8 else "_cache") for n in "kv"]
            for name in names:
                y[name] = x[name].clone()
                for s in (120, 30) if swa else (120,):      # 30: before every window, behind the sink
                    y[name][int(x["table"][0, s // 16]), :, s % 16] = bad
            out, lse = run_chunks(prm, y)
            rows = torch.ones(61, dtype=torch.bool, device=DEV)
            for j in range(60):
                t = 90 + j
                if t >= 120 and (not swa or t - 120 < swa):
                    rows[j] = False
            assert torch.equal(out[rows], want[0][rows]) and torch.equal(lse[rows], want[1][rows])
            hit = torch.ones((int((~rows).sum()), 4), dtype=torch.bool, device=DEV)
            if fp8 and bad == INF:      # an infinite scale makes a score below 0 -inf: that head does not see the position
                code = x["k_cache"].view(torch.uint8)[int(x["table"][0, 120 // 16]), :, 120 % 16].view(torch.float8_e4m3fn).double()
                hit = (x["q"][~rows].double() * code.repeat_interleave(2, 0)).sum(-1) > 0
            assert not torch.isfinite(out[~rows][hit]).any()


def test_equals_the_decode_attention():
    """Equal numbers of new tokens: what lsa_decode_attn gives, within both kernels' roundings; and out and lse are optional."""
    prm = P(16, 4)
    x = chunks(prm, [4] * 5, [4, 100, 64, 1000, 333], 64, seed=3)
    out, lse = run_chunks(prm, x)
    check_chunks(prm, x, out, lse)
    o2, l2 = lsa.decode_attn(prm, x["q"], x["k_cache"], x["v_cache"], x["ctx"], page_table=x["table"], rows_per_seq=4)
    # (each output is within 2^-7 of a sum that its largest value bounds in turn: 4 * 2^-7 of the largest |v| is beyond both)
    assert (out.float() - o2.float()).abs().max() <= 2.0 ** -5 * x["v_cache"].float().nan_to_num().abs().max()
    assert (lse - l2).abs().max() < 1e-3
    o3, l3 = lsa.chunk_attn(prm, x["q"], x["k_cache"], x["v_cache"], x["cu"], x["ctx"], page_table=x["table"], lse=None)
    assert l3 is None and torch.equal(o3, out)


def test_without_a_table_and_one_head():
    """Sequence b has page b alone; caches without the head dimension."""
    prm = P(4, 1, 64)
    x = chunks(prm, [10, 40], [50, 64], 64, seed=4, slack=0)
    order = x["table"][:, 0].long()
    y = dict(x, table=None, k_cache=x["k_cache"][order].contiguous(), v_cache=x["v_cache"][order].contiguous())
    a, b = run_chunks(prm, x), run_chunks(prm, y)
    z = dict(y, k_cache=y["k_cache"][:, 0], v_cache=y["v_cache"][:, 0])
    c = run_chunks(prm, z)
    check_chunks(prm, y, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(b[0], c[0])


def test_many_sequences():
    g = torch.Generator().manual_seed(6)
    new = torch.randint(0, 9, (200,), generator=g).tolist()
    ctx = [n + int(torch.randint(0, 300, (1,), generator=g)) for n in new]
    prm = P(8, 2, 64)
    x = chunks(prm, new, ctx, 16, seed=6)
    check_chunks(prm, x, *run_chunks(prm, x))


def test_same_bits_on_other_streams():
    prm = P(32, 8, 128, True)
    x = chunks(prm, [16, 200], [8000, 300], 64, seed=7)
    want = run_chunks(prm, x)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(s):
            got += [run_chunks(prm, x) for _ in range(2)]
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])


@pytest.mark.parametrize("tokens,ctx", [(12, 6000), (700, 1500)])
def test_in_a_graph(tokens, ctx):
    """Captured once, replayed over other caches, offsets and lengths."""
    prm = P(8, 2)
    x = chunks(prm, [tokens, 0], [ctx, ctx], 64, seed=8)
    for n in "kv":
        x[n + "_cache"].nan_to_num_()
    ws = torch.empty(max(1, lsa.chunk_attn_workspace_size(prm, 2, tokens, x["table"].shape[1], 64)), dtype=torch.uint8, device=DEV)
    out, lse = run_chunks(prm, x, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsa.chunk_attn(prm, x["q"], x["k_cache"], x["v_cache"], x["cu"], x["ctx"], page_table=x["table"], out=out, lse=lse, workspace=ws)
    for a, c0, c1 in ((tokens // 3, ctx, ctx - 70), (1, 1, ctx), (tokens - 1, tokens, 0)):
        x["q"].normal_(0, 2)
        x["k_cache"].normal_()
        x["cu"].copy_(i32([0, a, tokens]))
        x["ctx"].copy_(i32([c0, c1]))
        graph.replay()
        want = run_chunks(prm, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        check_chunks(prm, dict(x, new=[a, tokens - a], ctx_list=[c0, c1], at=[0, a, tokens]), out, lse)
