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
