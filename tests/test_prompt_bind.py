"""The compiled host side of the prompt-side operators beside the checks in Python: good calls pass it without them and give what
the calls behind them give; anything else is left to them."""
from __future__ import annotations

import os
import types

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_serve_bind import _append_call

pytestmark = pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")
DEV = "cuda"
BF = torch.bfloat16
NAMES = ("cache_append", "norm_append", "cache_read", "prefill_attn", "chunk_attn", "decode_attn")


def _normal(*shape, dtype=BF):
    return torch.randn(shape, device=DEV).to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _norm_call(kind):
    prm, a = _append_call(kind)
    if prm.n_heads:
        a["q_weight"] = _normal(prm.d_k - (prm.rot_dim if "q_rot" in a else 0))
    a.update(k_weight=_normal(prm.d_k - (prm.rot_dim if "k_rot" in a else 0)), k_out=kind != "keys", eps=1e-5)
    if kind == "placed":
        a["k_out"] = torch.zeros((6, prm.n_kv_heads, prm.d_k), dtype=BF, device=DEV)
    return prm, a


def _read_call(kind):
    fp8, one = kind == "fp8", kind == "latent"
    shape = (6, 16, 96) if one else (6, 2, 16, 64)
    cache = lambda: torch.randint(0, 100, shape, device=DEV).to(torch.uint8) if fp8 else _normal(*shape)
    a = dict(k_cache=cache(), cu=_i32([0, 20, 50]), n_tok=50, page_table=_i32([[5, 1, 0], [2, 3, 4]]))
    if not one:
        a["v_cache"] = cache()
    if fp8:
        a.update({n: torch.rand(shape[:3], device=DEV) for n in ("k_scale", "v_scale")})
    if kind == "given":
        a.update(start=_i32([3, 1]), k_out=_normal(50, 2, 64), v_out=_normal(50, 2, 64))
    return (lsa.CacheReadParams(1, 96) if one else lsa.CacheReadParams(2, 64, 64, fp8)), a


def _prefill_call(kind):
    n, m = (40, 3000) if kind == "cut" else (40, 60)
    fused = _normal(m, 8 * 64)
    a = dict(q=_normal(n, 4, 64), k=fused[:, :128].unflatten(1, (2, 64)), v=fused[:, 128:256].unflatten(1, (2, 64)), cu_q=_i32([0, 10, n]),
             cu_kv=_i32([0, 15, m]))
    prm = lsa.PrefillAttnParams(4, 2, 64, 64, 0.1)
    if kind == "own keys":
        a.update(k=a["k"][:n], v=a["v"][:n])
        del a["cu_kv"]
    if kind == "given":
        a.update(out=_normal(n, 4, 64), lse=torch.zeros((n, 4), device=DEV))
    if kind == "no lse":
        a.update(lse=False)
    if kind == "cut":
        a["workspace"] = torch.empty(lsa.prefill_attn_workspace_size(prm, 2, n, m), dtype=torch.uint8, device=DEV)
        assert a["workspace"].numel() > 0
    return prm, a


def _chunk_call(kind):
    fp8, width = kind == "fp8", 64 if kind == "cut" else 4
    shape = (128, 64, 64) if kind == "one head" else (128, 2, 64, 64)
    cache = lambda: torch.randint(0, 100, shape, device=DEV).to(torch.uint8) if fp8 else _normal(*shape)
    a = dict(q=_normal(30, 4, 64), k_cache=cache(), v_cache=cache(), cu_q=_i32([0, 7, 30]), ctx_len=_i32([100, width * 64]),
             page_table=torch.arange(2 * width, dtype=torch.int32, device=DEV).view(2, width))
    if fp8:
        a.update(k_scale=torch.rand(shape[:3], device=DEV), v_scale=torch.rand(shape[:3], device=DEV))
    prm = lsa.DecodeAttnParams(4, 1 if kind == "one head" else 2, 64, 64, False, 0.1, fp8)
    if kind == "given":
        a.update(out=_normal(30, 4, 64), lse=torch.zeros((30, 4), device=DEV))
    if kind == "cut":
        a["workspace"] = torch.empty(lsa.chunk_attn_workspace_size(prm, 2, 30, width, 64), dtype=torch.uint8, device=DEV)
        assert a["workspace"].numel() > 0
    return prm, a


def _both(monkeypatch, call, outputs):
    """Outputs of a good call with the checks in Python out of reach, and of the same call through them."""
    def none(*a, **kw):
        raise AssertionError("a good call reached the checks in Python")
    with monkeypatch.context() as m:
        m.setattr(lsa, "_need", none)
        first = [None if t is None else t.clone() for t in outputs(call())]
    with monkeypatch.context() as m:
        m.setattr(lsa, "_serve", types.SimpleNamespace(**{n: lambda *a: None for n in NAMES}))
        second = outputs(call())
    assert [t is None for t in first] == [t is None for t in second]
    for a, b in zip(first, second):
        assert a is None or torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gqa", "fp8", "latent", "placed", "keys"])
def test_norm_appends(monkeypatch, kind):
    torch.manual_seed(1)
    prm, a = _norm_call(kind)
    caches = [a.get(n) for n in ("k_cache", "v_cache", "k_scale", "v_scale")]

    def call():
        for t in caches:
            if t is not None:
                t.zero_()
        return lsa.norm_append(prm, **a)
    _both(monkeypatch, call, lambda r: [*r, *caches])
    assert caches[0].count_nonzero() > 0


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gqa", "fp8", "latent", "given"])
def test_reads(monkeypatch, kind):
    torch.manual_seed(2)
    prm, a = _read_call(kind)
    _both(monkeypatch, lambda: lsa.cache_read(prm, **a), lambda r: list(r))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["plain", "own keys", "given", "no lse", "cut"])
def test_prefills(monkeypatch, kind):
    torch.manual_seed(3)
    prm, a = _prefill_call(kind)
    _both(monkeypatch, lambda: lsa.prefill_attn(prm, **a), lambda r: list(r))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["plain", "fp8", "one head", "given", "cut"])
def test_chunks(monkeypatch, kind):
    torch.manual_seed(4)
    prm, a = _chunk_call(kind)
    _both(monkeypatch, lambda: lsa.chunk_attn(prm, **a), lambda r: list(r))


@pytest.mark.gpu
def test_what_is_not_as_it_should_be_is_refused():
    """The binding leaves it to the checks in Python, which say what it is; nothing is written."""
    torch.manual_seed(5)
    prm, a = _prefill_call("given")
    a["out"].zero_()
    for kw in (dict(q=a["q"].float()), dict(q=a["q"][:, :3]), dict(q=a["q"].cpu()), dict(k=a["k"][:, :1]), dict(v=a["v"][:50]), dict(v=None),
               dict(k=a["k"].transpose(0, 1)), dict(cu_q=a["cu_q"].long()), dict(cu_q=a["cu_q"][:0]), dict(cu_kv=a["cu_kv"][:2]), dict(cu_kv=None),
               dict(out=a["out"][:5]), dict(lse=a["lse"].double()), dict(q=3)):
        with pytest.raises((ValueError, lsa.LSAError)):
            lsa.prefill_attn(prm, **{**a, **kw})
    prm2, b = _chunk_call("given")
    b["out"].zero_()
    for kw in (dict(q=b["q"][:, :, :32]), dict(k_cache=b["k_cache"].float()), dict(v_cache=b["v_cache"][:5]), dict(v_cache=None), dict(k_scale=b["lse"]),
               dict(ctx_len=b["ctx_len"][:1]), dict(ctx_len=None), dict(page_table=b["page_table"].t()),
               dict(page_table=None, k_cache=b["k_cache"][:1], v_cache=b["v_cache"][:1]), dict(cu_q=b["cu_q"][:2]), dict(out=b["q"].float())):
        with pytest.raises((ValueError, lsa.LSAError)):
            lsa.chunk_attn(prm2, **{**b, **kw})
    prm3, c = _read_call("given")
    c["k_out"].zero_()
    for kw in (dict(n_tok=49), dict(n_tok=-1), dict(n_tok=1 << 40), dict(cu=c["cu"][:2]), dict(start=c["cu"]), dict(v_cache=None), dict(k_out=c["v_out"][:3]),
               dict(k_scale=c["start"])):
        with pytest.raises((ValueError, lsa.LSAError)):
            lsa.cache_read(prm3, **{**c, **kw})
    prm4, d = _norm_call("gqa")
    for kw in (dict(q_weight=d["q_weight"][:32]), dict(k_weight=d["k_weight"].float()), dict(eps=0.0), dict(eps=-1.0), dict(k_out=d["k_weight"]), dict(k_weight=3)):
        with pytest.raises((ValueError, lsa.LSAError)):
            lsa.norm_append(prm4, **{**d, **kw})
    assert a["out"].count_nonzero() == 0 and b["out"].count_nonzero() == 0 and c["k_out"].count_nonzero() == 0 and d["k_cache"].count_nonzero() == 0


@pytest.mark.gpu
def test_a_workspace_that_is_too_small_is_refused():
    for make, call in ((_prefill_call, lsa.prefill_attn), (_chunk_call, lsa.chunk_attn)):
        prm, a = make("cut")
        a["workspace"] = a["workspace"][:-256]
        with pytest.raises(lsa.LSAError, match="workspace"):
            call(prm, **a)
        big = torch.empty(a["workspace"].numel() + 512, dtype=torch.uint8, device=DEV)
        a["workspace"] = big[16:]          # not aligned
        with pytest.raises(lsa.LSAError, match="aligned"):
            call(prm, **a)


def test_other_arguments_are_left_to_python():
    x = torch.zeros((2, 1, 64), dtype=BF)
    s = lsa._serving()
    assert s.norm_append() is None and s.norm_append(*[None] * 23) is None
    assert s.cache_read(*[None] * 11) is None and s.prefill_attn(*[None] * 9) is None and s.chunk_attn(*[None] * 12) is None
    assert s.cache_read(lsa.CacheReadParams(1, 64), x, x, 3, *[None] * 7) is None
    assert s.prefill_attn(lsa.PrefillAttnParams(1, 1, 64, 64, 0.1), x, x, x, x, *[None] * 4) is None
