"""lsa_prefill_attn against 64 bits: packed prompts over packed keys and values. Tolerances: tests/prompt_check.py."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.prompt_check import BF16, DEV, check_prompts, i32, prompts, run_prompts

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def P(H, nk, d=128, dv=None, **kw):
    return lsa.PrefillAttnParams(H, nk, d, dv or min(d, 128), d ** -0.5, **kw)


EDGES = [1, 0, 2, 31, 32, 33, 63, 64, 65, 127, 129, 0, 255, 257, 700]
FORMS = [(32, 8), (16, 1), (4, 4, 64), (28, 4, 64), (40, 5), (100, 1), (1, 1), (6, 6, 192), (12, 4, 192), (96, 2, 64)]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_forms_and_lengths(form, causal):
    """Every head layout at prompts from none to several hundred tokens, at and around the tile sizes, in one call."""
    prm = P(*form, causal=causal)
    x = prompts(prm, EDGES, EDGES, seed=1)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("form", [(32, 8), (4, 4, 64), (6, 6, 192)], ids=str)
def test_last_parts_of_prompts(form):
    """Fewer tokens than keys (the rest was computed before), one token, more tokens than keys (the first ones see nothing), no keys."""
    prm = P(*form)
    x = prompts(prm, [1, 5, 130, 64, 40, 3, 0, 300], [1000, 5, 777, 65, 10, 0, 50, 301], seed=2)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("form", [(8, 2), (3, 3, 64), (4, 4, 192)], ids=str)
@pytest.mark.parametrize("sink,swa", [(0, 1), (4, 128), (0, 64), (100, 33), (64, 64), (0, 2000), (700, 100), (1, 65)])
def test_windows(form, sink, swa):
    prm = P(*form, k_sink=sink, k_swa=swa)
    x = prompts(prm, [1, 64, 130, 777, 5], [1, 64, 200, 777, 1500], seed=sink + swa)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("form", [(32, 8), (16, 1), (8, 8, 64), (16, 16, 192)], ids=str)
@pytest.mark.parametrize("n", [4099, 2048])
def test_long_prompts(form, n):
    prm = P(*form)
    x = prompts(prm, [n], [n], seed=n)
    check_prompts(prm, x, *run_prompts(prm, x))


@pytest.mark.parametrize("d", [64, 128, 192])
def test_slices_of_a_projection(d):
    """q, k and v as slices of one fused projection, rows of no sequence around the prompts (they hold NaN, and stay as they were)."""
    prm = P(6, 2, d)
    x = prompts(prm, [70, 1, 300], [70, 1, 300], seed=d, lead=3, tail=5, fused=True)
    out, lse = run_prompts(prm, x)
    check_prompts(prm, x, out, lse)
    y = dict(x, q=x["q"].contiguous(), k=x["k"].contiguous(), v=x["v"].contiguous())
    o2, l2 = run_prompts(prm, y)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    o3, l3 = lsa.prefill_attn(prm, x["q"], x["k"], x["v"], x["cu_q"], lse=False)       # the keys are the tokens'
    assert l3 is None and torch.equal(o3[3:-5], out[3:-5])


@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("sink,swa", [(0, 0), (4, 40)])
def test_what_is_not_attended_to_has_no_effect(d, sink, swa):
    """NaN and infinities in keys and values of later positions, of positions before the window and of neighbouring sequences."""
    prm = P(4, 2, d, k_sink=sink, k_swa=swa)
    x = prompts(prm, [150, 90, 200], [150, 90, 200], seed=d)
    want = run_prompts(prm, x)
    check_prompts(prm, x, *want)
    for bad in (NAN, INF, -INF):
        y = dict(x, k=x["k"].clone(), v=x["v"].clone())
        for at in (100, 240 + 77):          # token 100 of the first prompt, token 77 of the last
            y["k"][at], y["v"][at] = bad, bad
        y["v"][149, 1, 3] = bad             # the first prompt's last
        out, lse = run_prompts(prm, y)
        rows = torch.ones(440, dtype=torch.bool, device=DEV)
        for first, at, last in ((0, 100, 150), (240, 317, 440)):      # rows that do attend to it
            for r in range(at, last):
                if not swa or r - at < swa or at - first < sink:
                    rows[r] = False
        rows[149] = False
        assert torch.equal(out[rows], want[0][rows]) and torch.equal(lse[rows], want[1][rows]), bad
        assert not torch.isfinite(out[100]).any() and not torch.isfinite(out[317]).any()
        # (the value that only the last token of the first prompt has not finite)
        assert torch.isnan(out[149, 2:, 3]).all() if bad != bad else not torch.isfinite(out[149, 2:, 3]).any()


def test_values_that_are_not_finite_reach_their_rows():
    """An infinite value makes the outputs of the rows that attend to it infinite in that dimension alone, two of both signs NaN."""
    prm = P(2, 1, 64)
    x = prompts(prm, [130], [130], seed=3)
    want, _ = run_prompts(prm, x)
    x["v"][70, 0, 5], x["v"][90, 0, 5], x["v"][20, 0, 6] = INF, -INF, NAN
    out, _ = run_prompts(prm, x)
    assert (out[70:90, :, 5] == INF).all() and torch.isnan(out[90:, :, 5]).all() and torch.isnan(out[20:, :, 6]).all()
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[70:, :, 5] = False
    keep[20:, :, 6] = False
    assert torch.equal(out[keep], want[keep])


def test_scores_without_a_finite_maximum():
    """Every score -inf: o = 0, lse = -inf. Scores of 2^40 and more: the largest wins. NaN queries: their rows alone."""
    prm = P(2, 1, 128)
    x = prompts(prm, [100, 100, 100], [100, 100, 100], seed=4)
    x["q"][:100] = x["q"][:100].abs() + 0.1
    x["k"][:100] = -INF
    x["q"][150] = NAN
    x["q"][200:] *= 2.0 ** 20
    x["k"][200:] *= 2.0 ** 20
    out, lse = run_prompts(prm, x)
    assert (out[:100] == 0).all() and (lse[:100] == -INF).all()
    assert torch.isnan(out[150]).all() and torch.isfinite(out[100:150]).all() and torch.isfinite(out[151:200]).all()
    s = torch.matmul(x["q"][200:].double().transpose(0, 1), x["k"][200:, 0].double().T)
    s.masked_fill_(~torch.ones(100, 100, dtype=torch.bool, device=DEV).tril(), -INF)
    top = s.argmax(-1)                                                 # [heads, rows]
    assert torch.equal(out[200:], x["v"][200:, 0][top].transpose(0, 1))
    assert ((lse[200:].double() - s.amax(-1).T * prm.sm_scale).abs() <= 2.0 ** -15 * lse[200:].abs()).all()


def test_offsets_out_of_range():
    """Ranges beyond the tensors or backwards: no tokens, or no keys; other sequences are as they should be."""
    prm = P(4, 2, 64)
    x = prompts(prm, [50, 60, 70], [50, 60, 70], seed=5)
    want, wl = run_prompts(prm, x)
    y = dict(x, cu_kv=i32([0, 50, 181, 180]))          # the second ends behind the last row, the third backwards: no keys
    out, lse = run_prompts(prm, y)
    assert torch.equal(out[:50], want[:50]) and (out[50:] == 0).all() and (lse[50:] == -INF).all()
    for cu in ([-1, 50, 110, 181], [0, -5, 110, 2 ** 31 - 1], [60, 50, 110, 100]):
        y = dict(x, cu_q=i32(cu))
        out, lse = run_prompts(prm, y)
        for b in range(3):
            ok = 0 <= cu[b] <= cu[b + 1] <= 180
            if ok and cu[b + 1] - cu[b] == x["n_q"][b] and cu[b] == x["at"][b]:
                assert torch.equal(out[cu[b]:cu[b + 1]], want[cu[b]:cu[b + 1]])
        covered = torch.zeros(180, dtype=torch.bool, device=DEV)
        for b in range(3):
            if 0 <= cu[b] <= cu[b + 1] <= 180:
                covered[cu[b]:cu[b + 1]] = True
        assert (out[~covered] == 7.0).all()


def test_many_sequences():
    """More sequences than a wave scans at a time, most of them short."""
    g = torch.Generator().manual_seed(6)
    n = torch.randint(0, 40, (300,), generator=g).tolist()
    n[200] = 500
    prm = P(4, 2, 64)
    x = prompts(prm, n, n, seed=6)
    check_prompts(prm, x, *run_prompts(prm, x))


def test_nothing_to_do():
    prm = P(4, 2, 64)
    e = torch.empty((0, 4, 64), dtype=BF16, device=DEV)
    out, lse = lsa.prefill_attn(prm, e, e[:, :2], e[:, :2], i32([0, 0]))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    q = torch.randn((5, 4, 64), device=DEV).to(BF16)
    out, lse = lsa.prefill_attn(prm, q, e[:, :2], e[:, :2], i32([0, 5]), i32([0, 0]))      # no keys at all
    assert (out == 0).all() and (lse == -INF).all()


def test_same_call_same_bits_on_other_streams():
    prm = P(32, 8)
    x = prompts(prm, [300, 1000], [300, 1000], seed=8)
    want = run_prompts(prm, x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append([run_prompts(prm, x) for _ in range(2)])
    torch.cuda.synchronize()
    for pairs in got:
        for o, l in pairs:
            assert torch.equal(o, want[0]) and torch.equal(l, want[1])


@pytest.mark.parametrize("tokens", [64, 1500])
def test_in_a_graph(tokens):
    """Captured once, replayed over other inputs and offsets."""
    prm = P(8, 2)
    x = prompts(prm, [tokens, 0], [tokens, 0], seed=9)
    ws = torch.empty(max(1, lsa.prefill_attn_workspace_size(prm, 2, tokens, tokens)), dtype=torch.uint8, device=DEV)
    out, lse = run_prompts(prm, x, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lsa.prefill_attn(prm, x["q"], x["k"], x["v"], x["cu_q"], x["cu_kv"], out=out, lse=lse, workspace=ws)
    for a in (tokens // 3, 1, tokens - 1):
        x["q"].normal_(0, 2)
        x["k"].normal_()
        x["cu_q"].copy_(i32([0, a, tokens]))
        x["cu_kv"].copy_(i32([0, a, tokens]))
        graph.replay()
        want = run_prompts(prm, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        check_prompts(prm, dict(x, n_q=[a, tokens - a], n_k=[a, tokens - a], at=[0, a, tokens], kv_at=[0, a, tokens]), out, lse)
