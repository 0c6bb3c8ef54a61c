"""The compiled host side of the serving operators (_serve) beside the checks in Python: good calls pass it without them and
give what the calls behind them give; anything else is left to them."""
from __future__ import annotations

import os
import types

import pytest
import torch

from paper_2608_01662_amd import lsa

pytestmark = pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")
DEV = "cuda"
BF = torch.bfloat16


def _normal(*shape, dtype=BF):
    return torch.randn(shape, device=DEV).to(dtype)


def _append_call(kind):
    """(params, arguments of cache_append) of two tokens for each of three sequences."""
    g = dict(page_table=torch.arange(6, dtype=torch.int32, device=DEV).view(3, 2), ctx_len=torch.tensor([2, 9, 30], dtype=torch.int32, device=DEV),
             rows_per_seq=2, rope=_normal(32, 32, dtype=torch.float32), rows=True)
    if kind == "latent":
        return lsa.AppendParams(4, 1, 96, 0, 64, 32, True), dict(g, k=_normal(6, 1, 64), k_rot=_normal(6, 1, 32), k_cache=torch.zeros((6, 16, 96), dtype=BF, device=DEV),
                                                                 q=_normal(6, 4, 64), q_rot=_normal(6, 4, 32))
    fused = _normal(6, 8 * 64)
    heads = lambda a, b: fused[:, 64 * a:64 * b].unflatten(1, (b - a, 64))
    fp8 = kind == "fp8"
    cache = lambda: torch.zeros((6, 2, 16, 64), dtype=torch.uint8 if fp8 else BF, device=DEV)
    g.update(k=heads(4, 6), v=heads(6, 8), q=heads(0, 4), k_cache=cache(), v_cache=cache())
    if fp8:
        g.update(k_scale=torch.zeros((6, 2, 16), device=DEV), v_scale=torch.zeros((6, 2, 16), device=DEV))
    if kind == "placed":
        del g["ctx_len"]
        g.update(pos=torch.tensor([0, 1, 7, 8, 28, 29], dtype=torch.int32, device=DEV), seq=torch.tensor([0, 0, 1, 1, 2, 2], dtype=torch.int32, device=DEV),
                 q_out=torch.zeros((6, 4, 64), dtype=BF, device=DEV), rows=torch.zeros(6, dtype=torch.int64, device=DEV))
    if kind == "keys":
        for name in ("v", "v_cache", "q"):
            del g[name]
        return lsa.AppendParams(0, 2, 64, 0, 0, 32), dict(g, rows=False)
    return lsa.AppendParams(4, 2, 64, 64, 0, 32, fp8=fp8), g


def _attn_call(kind):
    latent, fp8 = kind == "latent", kind == "fp8"
    H, nk, d, dv = (16, 1, 576, 512) if latent else (8, 2, 64, 64)
    long = kind == "cut"
    n_phys, page = 512, 64
    shape = (n_phys, page, d) if latent else (n_phys, nk, page, d)
    cache = (lambda: torch.randint(0, 100, shape, device=DEV).to(torch.uint8)) if fp8 else (lambda: _normal(*shape))
    a = dict(q=_normal(4, H, d), k_cache=cache(), v_cache=None if latent else cache(), rows_per_seq=2,
             ctx_len=torch.tensor([5, 16384 if long else 100], dtype=torch.int32, device=DEV),
             page_table=torch.arange(512 if long else 4, dtype=torch.int32, device=DEV).view(2, -1))
    if fp8:
        a.update(k_scale=torch.rand((n_phys, nk, page), device=DEV), v_scale=torch.rand((n_phys, nk, page), device=DEV))
    prm = lsa.DecodeAttnParams(H, nk, d, dv, latent, 0.1, fp8)
    if kind == "given":
        a.update(out=torch.zeros((4, H, dv), dtype=BF, device=DEV), lse=torch.zeros((4, H), device=DEV))
    if kind == "no lse":
        a.update(lse=False)
    if long:
        a.update(workspace=torch.empty(lsa.decode_attn_workspace_size(prm, 2, 2, 256, page), dtype=torch.uint8, device=DEV))
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
        m.setattr(lsa, "_serve", types.SimpleNamespace(cache_append=lambda *a: None, decode_attn=lambda *a: None))
        second = outputs(call())
    assert [t is None for t in first] == [t is None for t in second]
    for a, b in zip(first, second):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gqa", "fp8", "latent", "placed", "keys"])
def test_appends(monkeypatch, kind):
    torch.manual_seed(1)
    prm, a = _append_call(kind)
    caches = [a.get(n) for n in ("k_cache", "v_cache", "k_scale", "v_scale")]

    def call():
        for t in caches:
            if t is not None:
                t.zero_()
        return lsa.cache_append(prm, **a)
    _both(monkeypatch, call, lambda r: [*r, *caches])
    assert caches[0].count_nonzero() > 0


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gqa", "fp8", "latent", "cut", "given", "no lse"])
def test_attention(monkeypatch, kind):
    torch.manual_seed(2)
    prm, a = _attn_call(kind)
    _both(monkeypatch, lambda: lsa.decode_attn(prm, **a), lambda r: list(r))


@pytest.mark.gpu
def test_what_is_not_as_it_should_be_launches_nothing():
    torch.manual_seed(3)
    prm, a = _append_call("gqa")
    order = ("k", "k_cache", "page_table", "ctx_len", "pos", "seq", "rows_per_seq", "n_seq", "rope", "k_rot", "v", "v_cache", "k_scale", "v_scale", "q", "q_rot",
             "q_out", "rows")
    bind = lambda **kw: lsa._serving().cache_append(prm, *[{**a, **kw}.get(n) for n in order])
    for kw in (dict(k=a["k"].float()), dict(k=a["k"][:5]), dict(k=a["k"].cpu()), dict(k=3), dict(v=None), dict(v_cache=a["v_cache"][:5]), dict(rope=None),
               dict(rope=a["rope"][:, :16]), dict(ctx_len=a["ctx_len"].long()), dict(ctx_len=a["ctx_len"][:2]), dict(pos=a["ctx_len"]), dict(rows_per_seq=3),
               dict(rows_per_seq=1 << 40), dict(rows_per_seq=None), dict(rows_per_seq=2.0), dict(n_seq=2), dict(k_scale=a["rope"]), dict(q_out=a["q"]),
               dict(page_table=a["page_table"].t()), dict(q=a["q"].transpose(0, 1)), dict(rows=1)):
        assert bind(**kw) is None, kw
    assert a["k_cache"].count_nonzero() == 0 and bind() is not None and a["k_cache"].count_nonzero() > 0


def test_host_tensors_and_other_arguments_are_left_to_python():
    x = torch.zeros((2, 1, 64), dtype=BF)
    s = lsa._serving()
    assert s.cache_append(lsa.AppendParams(0, 1, 64), x, x, *[None] * 4, 1, *[None] * 11) is None
    assert s.decode_attn(lsa.DecodeAttnParams(1, 1, 64, 64, False, 0.1), x, x, x, x, None, 1, *[None] * 5) is None
    assert s.cache_append() is None and s.cache_append(*[None] * 19) is None and s.decode_attn(*[None] * 12) is None


def test_missing_module_raises(monkeypatch, tmp_path):
    monkeypatch.setattr(lsa, "_serve", None)
    monkeypatch.setattr(lsa, "SERVE_PATH", str(tmp_path / "missing.so"))
    with pytest.raises(RuntimeError, match="missing"):
        lsa.decode_attn(None, None, None, None, None)
