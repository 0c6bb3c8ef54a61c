"""C-ABI checks of the prompt-side serving operators that need no GPU: arguments are refused on the host before any HIP
call (only pointers that fail validation are ever passed, so nothing reaches a device)."""
import ctypes
import os

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_serve_abi import A, FAKE, INVALID, ODD, OK, UNSUPPORTED

pytestmark = pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")


def norm_append(prm=A(8, 2, 128, 128, 0, 128), n_tok=4, norm=None, null=False, **kw):
    f = dict(q=FAKE if prm.n_heads else None, k=FAKE, v=FAKE if prm.d_v else None, q_stride=prm.n_heads * prm.d_k, q_rot_stride=0,
             k_stride=prm.n_kv_heads * prm.d_k, k_rot_stride=0, v_stride=prm.n_kv_heads * prm.d_v, rope=FAKE, rope_rows=64, ctx_len=FAKE,
             page_table=FAKE, q_out=FAKE + 4096 if prm.n_heads else None, k_cache=FAKE, v_cache=FAKE if prm.d_v else None)
    f.update(kw)
    t = lsa._AppendTensors(**f)
    an = dict(q_weight=None, k_weight=FAKE, eps=1e-6, k_out=None)
    an.update(norm or {})
    an = lsa._AppendNorm(**an)
    return lsa.lib().lsa_norm_append(ctypes.byref(prm.c()), None if null else ctypes.byref(an), ctypes.byref(t), n_tok, 4, 1, 8, 64, 100, None)


def test_norm_append_arguments():
    assert norm_append(null=True) == INVALID
    assert norm_append(n_tok=0, k=None) == OK
    for eps in (0.0, -1.0, float("inf"), float("nan"), 1e31):
        assert norm_append(norm=dict(eps=eps)) == INVALID
    assert norm_append(A(0, 2, 128, 128, 0, 128), norm=dict(q_weight=FAKE)) == INVALID       # norms of queries there are none of
    for x in ("q_weight", "k_weight", "k_out"):
        assert norm_append(norm={x: ODD}) == INVALID
        assert x in lsa.lib().lsa_last_error().decode()
    assert norm_append(norm=dict(k_out=FAKE), k_stride=512) == INVALID                       # in place, but not contiguous
    assert norm_append(k_stride=8) == INVALID and norm_append(q_out=ODD) == INVALID          # as lsa_cache_append
    assert norm_append(A(8, 2, 120, 128)) == UNSUPPORTED


def read(prm=lsa.CacheReadParams(8, 128, 128), n_tok=10, n_seq=2, max_pages=8, page=64, n_phys=100, null=False, **kw):
    f = dict(k=FAKE, ks=FAKE if prm.fp8 else None, v=FAKE if prm.d_v else None, vs=FAKE if prm.fp8 and prm.d_v else None, cu=FAKE, start=None,
             table=FAKE, k_out=FAKE, v_out=FAKE if prm.d_v else None)
    f.update(kw)
    return lsa.lib().lsa_cache_read(None if null else ctypes.byref(prm.c()), n_tok, n_seq, f["k"], f["ks"], f["v"], f["vs"], f["cu"], f["start"],
                                    f["table"], max_pages, page, n_phys, f["k_out"], f["v_out"], None)


R = lsa.CacheReadParams


def test_cache_read_arguments():
    assert read(null=True) == INVALID and read(R(0, 128)) == INVALID and read(R(5000, 128)) == INVALID
    for prm in (R(1, 0), R(1, 8), R(1, 24), R(1, 1040), R(1, 64, -16), R(1, 64, 24), R(1, 64, 1040)):
        assert read(prm) == UNSUPPORTED
    assert read(n_tok=0, k=None, cu=None) == OK and read(n_seq=0, k=None) == OK
    assert read(n_tok=-1) == INVALID and read(n_seq=-1) == INVALID and read(n_tok=1 << 28) == UNSUPPORTED
    assert read(max_pages=0) == INVALID and read(page=0) == INVALID and read(n_phys=0) == INVALID
    assert read(max_pages=1 << 26) == UNSUPPORTED and read(n_phys=1 << 23) == UNSUPPORTED
    assert read(table=None) == INVALID and read(table=None, max_pages=1, n_phys=1) == INVALID
    for x in ("k", "cu", "k_out", "v", "v_out"):
        assert read(**{x: None}) == INVALID
    assert read(ks=FAKE) == INVALID and read(R(8, 128, 128, True), ks=None) == INVALID and read(R(8, 128, 0, True), vs=FAKE) == INVALID
    assert read(R(8, 128), v=FAKE) == INVALID and read(R(8, 128), v_out=FAKE) == INVALID
    for x in ("k", "v", "k_out", "v_out"):
        assert read(**{x: FAKE + 8}) == INVALID
    for x in ("cu", "start", "table"):
        assert read(**{x: ODD}) == INVALID


def test_python_refusals():
    """What the binding refuses before the library is called (no tensor here is on a GPU)."""
    c = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lsa.cache_read(R(2, 64), c, torch.zeros(3, dtype=torch.int32), 5)
    with pytest.raises(ValueError):
        lsa.cache_read(R(2, 64), None, None, 5)
    with pytest.raises(ValueError):
        lsa.norm_append(A(0, 2, 64), torch.zeros((3, 2, 64), dtype=torch.bfloat16), c, k_out=True, pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        R(2 ** 31, 64).c()


def _prefill(prm=lsa.PrefillAttnParams(8, 2, 128, 128, 0.1), n_seq=2, n_tok=100, n_kv=100, null=False, ws=None, wsb=1 << 40, **kw):
    f = dict(q=FAKE, qs=prm.n_heads * prm.d_qk, k=FAKE, ks=prm.n_kv_heads * prm.d_qk, v=FAKE, vs=prm.n_kv_heads * prm.d_v, cu_q=FAKE,
             cu_kv=FAKE, out=FAKE, lse=FAKE)
    f.update(kw)
    return lsa.lib().lsa_prefill_attn(None if null else ctypes.byref(prm.c()), n_seq, n_tok, n_kv, f["q"], f["qs"], f["k"], f["ks"], f["v"],
                                      f["vs"], f["cu_q"], f["cu_kv"], f["out"], f["lse"], ws, wsb, None)


F = lsa.PrefillAttnParams


def test_prefill_attn_arguments():
    assert _prefill(null=True) == INVALID
    for prm in (F(8, 2, 128, 64, 0.1), F(8, 2, 192, 192, 0.1), F(8, 1, 576, 512, 0.1), F(8, 2, 96, 96, 0.1), F(8, 2, 64, 64, 0.1, False, 0, 5),
                F(8, 2, 64, 64, 0.1, False, 5, 0)):
        assert _prefill(prm) == UNSUPPORTED
    for prm in (F(8, 3, 64, 64, 0.1), F(0, 1, 64, 64, 0.1), F(8, 0, 64, 64, 0.1), F(1025, 1, 64, 64, 0.1), F(8, 2, 64, 64, 0.0),
                F(8, 2, 64, 64, float("nan")), F(8, 2, 64, 64, float("inf")), F(8, 2, 64, 64, 0.1, True, -1, 0), F(8, 2, 64, 64, 0.1, True, 0, -1),
                F(8, 2, 64, 64, 0.1, 2)):
        assert _prefill(prm) == INVALID
    assert _prefill(n_tok=0, q=None, cu_q=None) == OK and _prefill(n_seq=0, q=None, out=None) == OK
    assert _prefill(n_seq=-1) == INVALID and _prefill(n_tok=-1) == INVALID and _prefill(n_kv=-1) == INVALID
    assert _prefill(n_tok=1 << 27) == UNSUPPORTED and _prefill(n_seq=1 << 23) == UNSUPPORTED and _prefill(n_kv=1 << 31) == UNSUPPORTED
    assert _prefill(cu_kv=None, n_kv=99) == INVALID
    for x in ("q", "k", "v", "cu_q", "out"):
        assert _prefill(**{x: None}) == INVALID and _prefill(**{x: ODD}) == INVALID
    for x in ("cu_kv", "lse"):
        assert _prefill(**{x: ODD}) == INVALID
    for x, least in (("qs", 1024), ("ks", 256), ("vs", 256)):
        assert _prefill(**{x: least - 8}) == INVALID and _prefill(**{x: least + 4}) == INVALID and _prefill(**{x: 1 << 24}) == UNSUPPORTED


C = lsa.DecodeAttnParams


def _chunk(prm=C(8, 2, 128, 128, False, 0.1), n_seq=2, n_tok=100, max_pages=8, page=64, n_phys=100, null=False, ws=None, wsb=1 << 40, **kw):
    f = dict(q=FAKE, k=FAKE, ks=FAKE if prm.fp8 else None, v=FAKE, vs=FAKE if prm.fp8 else None, cu=FAKE, ctx=FAKE, table=FAKE, out=FAKE, lse=FAKE)
    f.update(kw)
    return lsa.lib().lsa_chunk_attn(None if null else ctypes.byref(prm.c()), n_seq, n_tok, f["q"], f["k"], f["ks"], f["v"], f["vs"], f["cu"],
                                    f["ctx"], f["table"], max_pages, page, n_phys, f["out"], f["lse"], ws, wsb, None)


def test_chunk_attn_arguments():
    assert _chunk(null=True) == INVALID
    for prm in (C(64, 1, 576, 512, True, 0.1), C(8, 2, 128, 64, False, 0.1), C(8, 2, 192, 128, False, 0.1), C(8, 2, 64, 64, True, 0.1)):
        assert _chunk(prm) == UNSUPPORTED
    for prm in (C(8, 3, 64, 64, False, 0.1), C(0, 1, 64, 64, False, 0.1), C(1025, 1, 64, 64, False, 0.1), C(8, 2, 64, 64, False, -1.0),
                C(8, 2, 64, 64, False, 0.1, False, -1), C(8, 2, 64, 64, 2, 0.1)):
        assert _chunk(prm) == INVALID
    assert _chunk(n_tok=0, q=None, cu=None) == OK and _chunk(n_seq=0, q=None, out=None) == OK
    assert _chunk(n_seq=-1) == INVALID and _chunk(n_tok=-1) == INVALID
    assert _chunk(n_tok=1 << 27) == UNSUPPORTED and _chunk(n_seq=1 << 23) == UNSUPPORTED
    assert _chunk(max_pages=0) == INVALID and _chunk(page=0) == INVALID and _chunk(n_phys=0) == INVALID
    assert _chunk(max_pages=1 << 26) == UNSUPPORTED and _chunk(n_phys=1 << 24) == UNSUPPORTED
    assert _chunk(table=None) == INVALID and _chunk(table=None, max_pages=1, n_phys=1) == INVALID
    for x in ("q", "k", "v", "cu", "ctx", "out"):
        assert _chunk(**{x: None}) == INVALID and _chunk(**{x: ODD}) == INVALID
    for x in ("table", "lse"):
        assert _chunk(**{x: ODD}) == INVALID
    assert _chunk(ks=FAKE) == INVALID and _chunk(C(8, 2, 64, 64, False, 0.1, True), vs=None) == INVALID


def test_attention_binding_refusals():
    """No tensor here is on a GPU, and numbers beyond 32 bits do not reach the C interface."""
    q = torch.zeros((5, 8, 64), dtype=torch.bfloat16)
    cu = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        lsa.prefill_attn(F(8, 2, 64, 64, 0.1), q, q[:, :2], q[:, :2], cu)
    with pytest.raises(ValueError):
        lsa.prefill_attn(F(8, 2, 64, 64, 0.1), None, None, None, None)
    with pytest.raises(ValueError):
        lsa.chunk_attn(C(8, 2, 64, 64, False, 0.1), q, q, q, cu, cu)
    with pytest.raises(ValueError):
        F(8, 2, 64, 64, 0.1, True, 0, 2 ** 32 + 5).c()
    with pytest.raises(ValueError):
        lsa.chunk_attn_workspace_size(C(8, 2, 64, 64, False, 0.1), 2 ** 32, 1, 1, 1)
