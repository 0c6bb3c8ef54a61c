"""C-ABI checks of the serving operators that need no GPU: arguments are refused on the host before any HIP
call (only pointers that fail validation are ever passed, so nothing reaches a device)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_01662_amd import lsa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE, ODD = 0x100000, 0x100002


def append(prm=lsa.AppendParams(8, 2, 128, 128, 0, 128), n_tok=4, n_seq=4, rps=1, max_pages=8, page=64, n_phys=100, null=False,
           **kw):
    fp8, dv, H = prm.fp8, prm.d_v, prm.n_heads
    f = dict(q=FAKE if H else None, q_rot=None, k=FAKE, k_rot=None, v=FAKE if dv else None, q_stride=H * prm.d_k, q_rot_stride=0,
             k_stride=prm.n_kv_heads * prm.d_k, k_rot_stride=0, v_stride=prm.n_kv_heads * dv,
             rope=FAKE if prm.rot_dim else None, rope_rows=64, seq=None, pos=None, ctx_len=FAKE, page_table=FAKE,
             q_out=FAKE + 4096 if H else None, k_cache=FAKE, k_scale=FAKE if fp8 else None, v_cache=FAKE if dv else None,
             v_scale=FAKE if fp8 and dv else None, rows=None)
    f.update(kw)
    t = lsa._AppendTensors(*[f[n] for n, _ in lsa._AppendTensors._fields_])
    return lsa.lib().lsa_cache_append(ctypes.byref(prm.c()), None if null else ctypes.byref(t), n_tok, n_seq, rps, max_pages,
                                      page, n_phys, None)


A = lsa.AppendParams


@pytest.mark.parametrize("prm,status", [
    (A(-1, 2, 128, 128), INVALID), (A(8, 0, 128, 128), INVALID), (A(8, 2, 120, 128), UNSUPPORTED), (A(8, 2, 1040, 128), UNSUPPORTED),
    (A(8, 2, 0, 128), UNSUPPORTED), (A(8, 2, 128, 24), UNSUPPORTED), (A(8, 2, 128, -16), UNSUPPORTED), (A(8, 2, 128, 128, 0, 8), UNSUPPORTED),
    (A(8, 2, 128, 128, 8, 16), UNSUPPORTED), (A(8, 2, 128, 128, 64, 80), INVALID), (A(8, 2, 128, 128, -16, 16), INVALID),
    (A(8, 2, 128, 128, 16, 2 ** 31 - 16), INVALID),
])
def test_append_parameters(prm, status):
    assert append(prm) == status


def test_append_arguments():
    L = lsa.lib()
    assert L.lsa_cache_append(None, None, 1, 1, 1, 1, 1, 1, None) == INVALID
    assert append(null=True) == INVALID
    assert append(n_tok=0, k=None, q=None, k_cache=None) == OK               # nothing to do, nothing touched
    assert append(n_tok=-1) == INVALID and append(n_tok=4, n_seq=-1) == INVALID and append(n_seq=0) == INVALID
    assert append(rps=0) == INVALID and append(page=0) == INVALID and append(max_pages=0) == INVALID and append(n_phys=0) == INVALID
    assert append(max_pages=1 << 26) == UNSUPPORTED                          # positions beyond int32
    assert append(n_phys=1 << 24) == UNSUPPORTED                             # rows of all heads beyond int32
    assert append(page_table=None) == INVALID                                # several pages without a table
    assert append(page_table=None, max_pages=1, n_phys=3) == INVALID         # fewer pages than sequences
    assert append(ctx_len=None) == INVALID and append(pos=FAKE) == INVALID   # exactly one of them
    assert append(n_tok=5) == INVALID and append(seq=FAKE) == INVALID        # by length: rows_per_seq of each
    assert append(rope=None) == INVALID and append(A(8, 2, 128, 128), rope=FAKE) == INVALID
    assert append(k_rot=FAKE, k_rot_stride=0) == INVALID                     # a stride below a token's elements
    assert append(A(8, 2, 128, 128, 0, 64), k_rot=FAKE, k_rot_stride=128) == INVALID      # rotated dims not the last
    for name in ("k", "v", "q", "q_out", "k_cache", "v_cache"):
        assert append(**{name: None}) == INVALID, name
        assert append(**{name: ODD}) == INVALID, name
    for name in ("k_stride", "v_stride", "q_stride"):
        assert append(**{name: 100}) == INVALID and append(**{name: 2052}) == INVALID, name
    assert append(k_scale=FAKE) == INVALID                                   # bf16 takes no scales
    fp8 = A(8, 2, 128, 128, 0, 128, False, True)
    assert append(fp8, k_scale=None) == INVALID and append(fp8, v_scale=None) == INVALID
    assert append(A(8, 1, 128), v=FAKE) == INVALID and append(A(8, 1, 128), v_cache=FAKE) == INVALID
    assert append(A(0, 2, 128, 128), q=FAKE) == INVALID and append(A(0, 2, 128, 128), q_rot=FAKE) == INVALID
    assert append(q_out=FAKE, q_stride=2048) == INVALID                      # in place only where q is contiguous
    assert append(rows=0x100004) == INVALID and append(ctx_len=ODD) == INVALID and append(rope=0x100004) == INVALID
    assert b"rope" in L.lsa_last_error()


D = lsa.DecodeAttnParams


def attn(prm=D(32, 8, 128, 128, False, 0.1), n_seq=4, rps=1, q=FAKE, k=FAKE, ks=None, v=FAKE, vs=None, ctx=FAKE, table=FAKE,
         max_pages=8, page=64, n_phys=100, out=FAKE, lse=None, ws=FAKE, wsb=1 << 40):
    return lsa.lib().lsa_decode_attn(ctypes.byref(prm.c()), n_seq, rps, q, k, ks, v, vs, ctx, table, max_pages, page, n_phys, out,
                                     lse, ws, wsb, None)


@pytest.mark.parametrize("prm,status", [
    (D(32, 5, 128, 128, False, 0.1), INVALID), (D(0, 1, 128, 128, False, 0.1), INVALID), (D(8, 0, 128, 128, False, 0.1), INVALID),
    (D(2048, 1, 128, 128, False, 0.1), INVALID), (D(8, 8, 96, 96, False, 0.1), UNSUPPORTED), (D(8, 8, 128, 64, False, 0.1), UNSUPPORTED),
    (D(64, 1, 576, 512, False, 0.1), UNSUPPORTED), (D(64, 2, 576, 512, True, 0.1), UNSUPPORTED), (D(64, 1, 576, 512, True, 0.1, True), UNSUPPORTED),
    (D(8, 8, 128, 128, False, 0.0), INVALID), (D(8, 8, 128, 128, False, float("inf")), INVALID), (D(8, 8, 128, 128, False, 0.1, k_sink=-1), INVALID),
    (D(8, 8, 128, 128, False, 0.1, k_swa=-1), INVALID),
])
def test_attention_parameters(prm, status):
    assert attn(prm) == status
    assert lsa.decode_attn_workspace_size(prm, 4, 1, 8, 64) == 0


def test_attention_arguments():
    L = lsa.lib()
    assert L.lsa_decode_attn(None, 1, 1, *[None] * 7, 1, 1, 1, None, None, None, 0, None) == INVALID
    assert attn(n_seq=0, q=None, k=None, v=None, ctx=None, out=None, ws=None, wsb=0) == OK
    assert attn(n_seq=-1) == INVALID and attn(rps=0) == INVALID and attn(max_pages=0) == INVALID and attn(page=0) == INVALID
    assert attn(rps=2000) == UNSUPPORTED and attn(max_pages=1 << 26) == UNSUPPORTED and attn(n_phys=1 << 24) == UNSUPPORTED
    assert attn(n_phys=0) != OK
    assert attn(table=None) == INVALID and attn(table=None, max_pages=1, n_phys=3) == INVALID
    for name in ("q", "k", "ctx", "out"):
        assert attn(**{name: None}) == INVALID, name
    for name in ("q", "k", "v", "out", "lse", "table", "ctx"):
        assert attn(**{name: 0x100001}) == INVALID, name
    assert attn(v=None) == INVALID and attn(ks=FAKE, vs=FAKE) == INVALID
    fp8 = D(32, 8, 128, 128, False, 0.1, True)
    assert attn(fp8) == INVALID and attn(fp8, ks=FAKE) == INVALID
    assert attn(D(64, 1, 576, 512, True, 0.1)) == INVALID                    # a latent cache takes no values
    # long contexts of few sequences are cut: the call needs room for the parts
    need = lsa.decode_attn_workspace_size(D(32, 8, 128, 128, False, 0.1), 1, 1, 2048, 64)
    if need:
        assert attn(n_seq=1, max_pages=2048, ws=None) == WORKSPACE and attn(n_seq=1, max_pages=2048, wsb=need - 1) == WORKSPACE
        assert attn(n_seq=1, max_pages=2048, ws=0x100080) == WORKSPACE


def test_binding_refuses_host_tensors():
    bf = dict(dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        lsa.cache_append(A(0, 1, 64), torch.zeros((2, 1, 64), **bf), torch.zeros((2, 16, 64), **bf), pos=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        lsa.decode_attn(D(1, 1, 64, 64, False, 0.1), torch.zeros((2, 1, 64), **bf), torch.zeros((2, 16, 64), **bf),
                        torch.zeros((2, 16, 64), **bf), torch.ones(2, dtype=torch.int32))


def test_exact_division_of_positions():
    """The kernels divide positions by the page size with one product and shift (fast_div): exact for every
    0 <= n < 2^31, checked at the multiples' neighbours, where a reciprocal too small or large would show."""
    text = open(os.path.join(ROOT, "paper_2608_01662_amd", "csrc", "launch.hpp")).read()
    assert re.search(r"shift = 31 \+ l;", text) and re.search(r"\(uint64_t\(1\) << shift\) / d \+ 1", text)
    for d in list(range(1, 1100)) + [4095, 4097, 65535, 65537, (1 << 30) - 1, (1 << 31) - 1]:
        l = 0
        while (1 << l) < d:
            l += 1
        shift, mul = 31 + l, (1 << (31 + l)) // d + 1
        top = (1 << 31) - 1
        assert mul < 1 << 33 and top * mul < 1 << 64
        for n in {0, 1, d - 1, d, d + 1, top, top // d * d, top // d * d - 1, top // 2 // d * d - 1, 12345678 // d * d - 1}:
            if 0 <= n <= top:
                assert (n * mul) >> shift == n // d, (n, d)


def test_attention_workspace():
    """Short tables need none; longer ones room for two fp32 partials per workgroup, of which there are no more than
    the GPU runs at once; calls of more tiles than the kernels count are refused."""
    size = lsa.decode_attn_workspace_size
    gqa, mla = D(32, 8, 128, 128, False, 0.1), D(64, 1, 576, 512, True, 0.1)
    assert size(gqa, 1, 1, 8, 64) == 0 and size(gqa, 64, 1, 32, 64) == 0 and size(mla, 256, 1, 20, 64) == 0
    assert size(gqa, 0, 1, 2048, 64) == 0
    for prm, cols in ((gqa, 16), (mla, 64), (D(32, 1, 128, 128, False, 0.1), 32)):
        part = cols * (prm.d_v + 2) * 4
        for n_seq, pages in ((1, 2048), (7, 500), (64, 2048), (300, 100)):
            assert 2 * part <= size(prm, n_seq, 1, pages, 64) <= 2 * 512 * part + n_seq * prm.n_kv_heads * 16 + 768, (cols, n_seq)
    # a window bounds the tiles, whatever the table
    assert size(D(32, 8, 128, 128, False, 0.1, k_sink=4, k_swa=256), 64, 1, 4096, 64) == 0
    assert attn(n_seq=4096, max_pages=1 << 19, n_phys=1 << 20) == UNSUPPORTED
    assert b"2^30" in lsa.lib().lsa_last_error()
