"""lsa_decode_attn at the end of the positions that 32 bits count: a context of 2^31 - 16 tokens, whose last tile begins at
2^31 - 32, through a table of pages that share a few physical ones.

The three new tokens have scores near 30 in the last page, so that what a row must not see would show. Against the definition
in 64 bits, with every cache row counted as often as it is seen. Tolerances of test_gpu_decode_attn, and for the others' weights,
e^-30 2^31 = 2^-12 of the sum and added in chains of at most 2^18 (each off by 2^-24 of what it has): 2^-18 more, 2^-14 allowed."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_gpu_decode_attn import GQA, MLA, _params

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
P, WIDTH = 16, (1 << 27) - 1
CTX = P * WIDTH
SHARED = 32     # physical pages of all but the last page


def _inputs(prm, R):
    g = torch.Generator(device=DEV).manual_seed(9)
    table = (torch.arange(WIDTH, device=DEV) % SHARED).to(torch.int32)[None]
    table[0, -1] = SHARED
    shape = (SHARED + 1, P, prm.d_qk) if prm.latent else (SHARED + 1, prm.n_kv_heads, P, prm.d_qk)
    q = torch.randn((R, prm.n_heads, prm.d_qk), generator=g, device=DEV).to(torch.bfloat16)
    q[..., 5] = 8.0
    x = dict(q=q, ctx=torch.tensor([CTX], dtype=torch.int32, device=DEV), table=table)
    for name in ["k"] + ([] if prm.latent else ["v"]):
        c = torch.randn(shape, generator=g, device=DEV)
        if name == "k":
            c[..., 5] = 0.0
            c[SHARED, ..., P - 3:, 5] = 30.0 / (8.0 * prm.sm_scale)
        if prm.fp8:
            s = c.abs().amax(-1) / 448
            x[name + "_scale"] = s
            c = (c / s[..., None]).to(torch.float8_e4m3fn)
        else:
            c = c.to(torch.bfloat16)
        x[name + "_cache"] = c
    return x


def _run(prm, x, R):
    return lsa.decode_attn(prm, x["q"], x["k_cache"], x.get("v_cache"), x["ctx"], page_table=x["table"], rows_per_seq=R,
                           k_scale=x.get("k_scale"), v_scale=x.get("v_scale"))


def _rows(x, name, prm):
    """The cache's rows [33 * 16, d] of the one head in 64 bits."""
    c = x[name + "_cache"].double()
    if prm.fp8:
        c = c * x[name + "_scale"].double()[..., None]
    return c.reshape(-1, c.shape[-1]).cpu()


def _counts(prm, t):
    """How often a query at position t sees each row."""
    n = torch.zeros((SHARED + 1, P), dtype=torch.float64)
    if prm.k_swa:
        for s in list(range(prm.k_sink)) + list(range(t - prm.k_swa + 1, t + 1)):
            pg = s // P
            n[SHARED if pg == WIDTH - 1 else pg % SHARED, s % P] += 1
        return n.reshape(-1)
    n[:SHARED] = (WIDTH - 1) // SHARED
    n[:(WIDTH - 1) % SHARED] += 1
    n[SHARED, :t % P + 1] = 1
    return n.reshape(-1)


@pytest.mark.parametrize("sink,swa", [(0, 0), (40, 100)], ids=["all", "window"])
@pytest.mark.parametrize("form", [(GQA, 4, 1, 64, False), (GQA, 24, 1, 128, True), (MLA, 20, 1, 576, False)], ids=str)
def test_the_last_tile(form, sink, swa):
    prm, R = _params(*form, k_sink=sink, k_swa=swa), 3
    x = _inputs(prm, R)
    out, lse = _run(prm, x, R)
    k = _rows(x, "k", prm)
    v = k[:, :prm.d_v] if prm.latent else _rows(x, "v", prm)
    q = x["q"].double().cpu()
    for j in range(R):
        n = _counts(prm, CTX - R + j)
        s = prm.sm_scale * (q[j] @ k.T) + n.log()
        top = s.amax(1, keepdim=True)
        p = (s - top).exp()
        total = p.sum(1, keepdim=True)
        o, spread, l = p @ v / total, p @ v.abs() / total, (total.log() + top)[:, 0]
        e = (prm.d_qk + 2) * 2.0 ** -23 * prm.sm_scale * float((q[j].abs() @ k.abs().T).max())
        assert ((out[j].double().cpu() - o).abs() <= (3 * 2.0 ** -8 + 2 * e + 2.0 ** -18 + 2.0 ** -14) * spread).all(), j
        assert ((lse[j].double().cpu() - l).abs() <= e + 2.0 ** -18 * (1 + l.abs()) + 2.0 ** -14).all(), j


@pytest.mark.parametrize("bad", [float("nan"), float("-inf")], ids=str)
@pytest.mark.parametrize("form", [(GQA, 4, 1, 64, False), (MLA, 20, 1, 576, False)], ids=str)
def test_a_value_of_the_newest_token_alone(form, bad):
    """A value of the newest token that is no number or infinite reaches its own row alone. (Latent: a -inf in its key, with
    a weight of 0, so that its row has NaN in that dim.)"""
    prm, R = _params(*form, k_sink=40, k_swa=100), 3
    x = _inputs(prm, R)
    x["q"][..., 7] = 1.0
    if prm.latent:
        x["k_cache"][SHARED, P - 1, 7] = -1e30
    ref, ref_l = (y.clone() for y in _run(prm, x, R))
    c = x["k_cache"][SHARED] if prm.latent else x["v_cache"][SHARED, 0]
    c[P - 1, 7] = float("-inf") if prm.latent else bad
    out, lse = _run(prm, x, R)
    assert torch.equal(out[:R - 1], ref[:R - 1]) and torch.equal(lse, ref_l)
    assert not torch.isfinite(out[R - 1][:, 7]).any()
    out[R - 1, :, 7] = ref[R - 1, :, 7]
    assert torch.equal(out, ref)
