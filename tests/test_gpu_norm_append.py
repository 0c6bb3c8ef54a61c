"""lsa_norm_append against the float64 oracle: norms of query and key heads, rotation, cached rows and keys beside the cache.

Tolerances, from the arithmetic (u = 2^-24): the squares of a head of up to 1024 values are summed without cancellation,
16 in a chain per lane and six exchanges, at most 22 u relative; mean, eps, root (which halves what came before),
reciprocal and the products with x and the weight add at most 12 u: a normed value is off by at most 24 u of itself. A rotated
value a c - b s is then off by at most 27 u (|a| + |b|) <= 54 u max|y|, and is rounded once to bf16: 2^-8 relative. An fp8 row:
the scale is off by at most 60 u relative, a code stands for its value within half a step of e4m3: 2^-4
relative, or 2^-10 of the scale below the normal range."""
from __future__ import annotations

import pytest
import torch

import oracle.serve_oracle as orc
from paper_2608_01662_amd import lsa
from tests.test_gpu_append import _caches, _dev_inputs, _i32, _setup

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U, EPS = 2.0 ** -24, 1e-5
A = lsa.AppendParams


def _weights(prm, s, seed, q=True, k=True):
    g = torch.Generator().manual_seed(100 + seed)
    cut = lambda part: prm.d_k - (prm.rot_dim if part in s else 0)
    make = lambda n: (1 + 0.3 * torch.randn(n, generator=g)).to(torch.bfloat16)
    return (make(cut("q_rot")) if q and prm.n_heads else None), (make(cut("k_rot")) if k else None)


def _want(prm, s, x, weight, t, turn=True):
    """(the head as rotated, the largest magnitude before) of token t in float64"""
    y = s[x][t].double()
    if weight is not None:
        y = orc.norm(y, weight.double(), EPS)
    if x + "_rot" in s:
        y = torch.cat([y, s[x + "_rot"][t].double()], 1)
    if not prm.rot_dim or not turn:
        return y, y.abs().amax(1, keepdim=True)
    return orc.rotate(y, prm.rot_start, prm.rot_dim, prm.interleaved, s["rope"][s["pos"][t]]), y.abs().amax(1, keepdim=True)


def _check(prm, s, wq, wk, c, q_out, k_out, rows):
    page = s["page"]
    n_pos = len(s["rope"]) if prm.rot_dim else 1 << 30
    ok = [0 <= b < len(s["lens"]) and 0 <= p < min(len(s["table"][0]) * page, n_pos) for b, p in zip(s["seq"], s["pos"])]
    want_rows = [orc.cache_row(b, p if o else -1, s["table"], page, len(s["lens"]), s["n_phys"]) for b, p, o in zip(s["seq"], s["pos"], ok)]
    assert rows.tolist() == want_rows

    def near(got, want, reach, t):
        tol = 1.01 * 2.0 ** -8 * want.abs() + 54 * U * reach
        assert ((got - want).abs() <= tol).all(), t
    for x, w, out, heads in (("q", wq, q_out, prm.n_heads), ("k", wk, k_out, prm.n_kv_heads)):
        if heads and out is not None:
            for t in range(s["n"]):
                want, reach = _want(prm, s, x, w, t) if ok[t] else (torch.zeros(heads, prm.d_k).double(), 0.0)
                near(out[t].double().cpu(), want, reach, (x, t))
    for x, d in (("k", prm.d_k), ("v", prm.d_v)):
        if not d:
            continue
        flat = c[x + "_cache"].transpose(1, 2).reshape(-1, prm.n_kv_heads, d).cpu()
        scales = c[x + "_scale"].transpose(1, 2).reshape(-1, prm.n_kv_heads).cpu() if prm.fp8 else None
        written = torch.zeros(flat.shape[0], dtype=torch.bool)
        for t, r in enumerate(want_rows):
            if r < 0:
                continue
            written[r] = True
            want, reach = _want(prm, s, x, wk, t) if x == "k" else (s["v"][t].double(), 0.0)
            if not prm.fp8:
                if x == "v":
                    assert torch.equal(flat[r], s["v"][t])
                else:
                    near(flat[r].double(), want, reach, (x, t))
                continue
            top = want.abs().amax(1)
            ws = torch.where(top > 0, (top / 448).clamp_min(2.0 ** -126), torch.ones_like(top))
            assert ((scales[r].double() - ws).abs() <= 60 * U * ws).all(), (x, t)
            got = flat[r].view(torch.float8_e4m3fn).double() * scales[r].double()[:, None]
            tol = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * ws[:, None]) * (1 + 2.0 ** -10) + 60 * U * reach
            assert ((got - want).abs() <= tol).all(), (x, t)
        assert (flat[~written] == (33 if prm.fp8 else 7.0)).all(), x      # what was not written is as it was
        if prm.fp8:
            assert (scales[~written] == 7.0).all(), x


def _call(prm, s, wq, wk, k_out=True, rope_rows=None, **kw):
    c, x = _caches(prm, s), _dev_inputs(s)
    to = lambda w: None if w is None else w.to(DEV)
    rope = None if s["rope"] is None else s["rope"][:rope_rows].to(DEV)
    r = lsa.norm_append(prm, x.pop("k"), c["k_cache"], q_weight=to(wq), k_weight=to(wk), eps=EPS, k_out=k_out,
                        page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]), rope=rope, rows=True, **x,
                        **{k: v for k, v in c.items() if k != "k_cache"}, **kw)
    return c, r


FORMS = [
    (A(8, 2, 128, 128, 0, 128, False, False), dict(fused=True)),
    (A(8, 2, 128, 128, 0, 64, True, True), dict(fused=True)),
    (A(5, 5, 64, 64, 0, 64, False, True), {}),
    (A(16, 1, 128, 128, 32, 96, True, False), dict(fused=True)),
    (A(3, 1, 80, 48, 16, 32, False, True), {}),           # heads of a number of units that is no power of two
    (A(3, 2, 80, 48, 16, 32, True, False), {}),
    (A(4, 2, 16, 1024, 0, 16, False, True), {}),          # the least and the greatest width
    (A(2, 1, 1024, 16, 0, 1024, True, False), {}),
    (A(4, 2, 64, 64), dict(fused=True)),                  # no rotation
    (A(0, 3, 64, 64, 0, 32, False, False), {}),           # no queries
    (A(64, 1, 576, 0, 512, 64, True, False), dict(split=True)),
    (A(2, 1, 576, 0, 512, 64, True, True), {}),
]


@pytest.mark.parametrize("prm,kw", FORMS, ids=lambda x: "-".join(str(v) for v in vars(x).values()) if hasattr(x, "d_k") else "")
@pytest.mark.parametrize("page", [64, 37])
def test_norm_append_forms(prm, kw, page):
    s = _setup(prm, [1, 70, 5, 131], [1, 3, 5, 31], page, seed=page, **kw)
    wq, wk = _weights(prm, s, page)
    c, (q, k, rows) = _call(prm, s, wq, wk)
    _check(prm, s, wq, wk, c, q, k, rows)


@pytest.mark.parametrize("q,k,k_out", [(True, False, True), (False, True, False), (False, False, True), (True, True, False)])
@pytest.mark.parametrize("fp8", [False, True])
def test_norms_are_optional(q, k, k_out, fp8):
    """Only queries, only keys or none normed; with and without keys beside the cache."""
    prm = A(6, 3, 80, 64, 0, 80, False, fp8)
    s = _setup(prm, [9, 40], [9, 5], 16, seed=3)
    wq, wk = _weights(prm, s, 3, q, k)
    c, (qo, ko, rows) = _call(prm, s, wq, wk, k_out=k_out)
    assert (ko is not None) == k_out
    _check(prm, s, wq, wk, c, qo, ko, rows)


def test_many_tokens_take_four_heads_a_thread():
    """A call of more than 2^18 units of queries: the form of large calls."""
    prm = A(32, 2, 128, 128, 0, 64, False, True)
    s = _setup(prm, [600, 700], [520, 600], 64, seed=4, fused=True)
    wq, wk = _weights(prm, s, 4)
    c, (q, k, rows) = _call(prm, s, wq, wk)
    _check(prm, s, wq, wk, c, q, k, rows)


def test_tokens_without_a_place():
    """Sequences, positions and angles out of range: queries and keys are zeros, nothing is cached; an unmapped page alone
    leaves the keys beside the cache as they should be."""
    prm = A(2, 2, 64, 64, 0, 64, False, False)
    s = _setup(prm, [100, 100, 100], [4, 4, 4], 16, seed=9)
    s["seq"][0], s["seq"][1], s["pos"][2] = -1, 3, -1
    s["pos"][3] = len(s["table"][0]) * 16
    s["table"][1][6] = -1
    s["table"][2][6] = s["n_phys"]
    wq, wk = _weights(prm, s, 9)
    c, (q, k, rows) = _call(prm, s, wq, wk)
    assert rows.tolist()[:12] == [-1] * 12
    _check(prm, s, wq, wk, c, q, k, rows)
    s["rope"] = s["rope"][:97]      # positions 97 .. 99 of sequence 1 have no angles
    c, (q, k, rows) = _call(prm, s, wq, wk)
    _check(prm, s, wq, wk, c, q, k, rows)


def test_in_place_and_given_outputs():
    """q_out and k_out may be the inputs themselves where those are contiguous; given tensors are the ones returned."""
    prm = A(4, 2, 64, 64, 0, 64, True, True)
    s = _setup(prm, [30, 7], [20, 7], 8, seed=5)
    wq, wk = _weights(prm, s, 5)
    c0, (q0, k0, r0) = _call(prm, s, wq, wk)
    c, x = _caches(prm, s), _dev_inputs(s)
    rows = torch.empty(s["n"], dtype=torch.int64, device=DEV)
    q, k, r = lsa.norm_append(prm, x["k"], c["k_cache"], q_weight=wq.to(DEV), k_weight=wk.to(DEV), eps=EPS, k_out=x["k"], q_out=x["q"],
                              q=x["q"], v=x["v"], rows=rows, page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                              rope=s["rope"].to(DEV), **{n: t for n, t in c.items() if n != "k_cache"})
    assert q is x["q"] and k is x["k"] and r is rows
    assert torch.equal(q, q0) and torch.equal(k, k0) and torch.equal(r, r0)
    for name in c:
        assert torch.equal(c[name], c0[name])


def test_zero_heads_and_large_values():
    """A head of zeros stays zeros; heads of 2^40 are normed as others are (their squares fit fp32)."""
    prm = A(2, 2, 64, 64, 0, 32, False, False)
    s = _setup(prm, [6], [6], 16, seed=6)
    s["q"][0], s["k"][1] = 0, 0
    s["q"][2] *= 2.0 ** 40
    s["k"][3] *= 2.0 ** 40
    wq, wk = _weights(prm, s, 6)
    c, (q, k, rows) = _call(prm, s, wq, wk)
    _check(prm, s, wq, wk, c, q, k, rows)
    assert (q[0] == 0).all() and (k[1] == 0).all()


def test_decode_form_in_a_graph():
    """The tokens named by context lengths, captured once and replayed over other inputs and lengths."""
    prm = A(8, 2, 128, 128, 0, 128, False, True)
    g = torch.Generator().manual_seed(8)
    table = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    rope = torch.randn((256, 128), generator=g).to(DEV)
    wq, wk = (torch.randn(128, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    fused = torch.zeros((3, 12 * 128), dtype=torch.bfloat16, device=DEV)
    ctx = torch.ones(3, dtype=torch.int32, device=DEV)
    make = lambda: {x + "_cache": torch.zeros((12, 2, 64, 128), dtype=torch.uint8, device=DEV) for x in "kv"} | \
        {x + "_scale": torch.zeros((12, 2, 64), device=DEV) for x in "kv"}
    heads = lambda a, b: fused[:, 128 * a:128 * b].unflatten(1, (b - a, 128))

    def call(c):
        return lsa.norm_append(prm, heads(8, 10), c["k_cache"], v=heads(10, 12), q=heads(0, 8), q_weight=wq, k_weight=wk, eps=EPS, k_out=True,
                               rope=rope, page_table=table, ctx_len=ctx, rows=True, **{n: t for n, t in c.items() if n != "k_cache"})
    a, b = make(), make()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(a)
    torch.cuda.synchronize()
    for t in a.values():
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(a)
    for step in range(3):
        fused.copy_(torch.randn(fused.shape, generator=g).to(torch.bfloat16))
        ctx.copy_(torch.tensor([1 + step, 64 + step, 256 - 2 + step], dtype=torch.int32))   # (the last one's end: beyond the table)
        graph.replay()
        want = call(b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert all(torch.equal(a[n], b[n]) for n in a)


def test_no_tokens_and_another_stream():
    prm = A(2, 1, 64, 64, 0, 64, False, False)
    s = _setup(prm, [5], [5], 16, seed=7)
    wq, wk = _weights(prm, s, 7)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        c, (q, k, rows) = _call(prm, s, wq, wk)
    st.synchronize()
    _check(prm, s, wq, wk, c, q, k, rows)
    x = torch.empty((0, 1, 64), dtype=torch.bfloat16, device=DEV)
    q, k, rows = lsa.norm_append(prm, x, c["k_cache"], q=x.new_empty((0, 2, 64)), v=x, v_cache=c["v_cache"], pos=_i32([]), seq=_i32([]),
                                 page_table=_i32(s["table"]), rope=s["rope"].to(DEV), q_weight=wq.to(DEV), k_weight=wk.to(DEV), k_out=True)
    assert q.shape == (0, 2, 64) and k.shape == (0, 1, 64) and rows is None
