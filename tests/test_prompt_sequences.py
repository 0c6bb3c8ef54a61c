"""The most sequences of a call of lsa_prefill_attn and lsa_chunk_attn: every workgroup looks through all of them, so that a call's time grows with their
square, and the sums over sequences (of whatever offsets the device holds) have to stay within 31 bits."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_prompt_abi import C, F, INVALID, UNSUPPORTED, _chunk, _prefill

pytestmark = pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")
MOST = 1 << 16


def test_more_sequences_are_refused():
    for call in (_prefill, _chunk):
        assert call(n_seq=MOST, q=None) == INVALID      # (the next check refuses it)
        for n in (MOST + 1, 1 << 20):
            assert call(n_seq=n) == UNSUPPORTED and "n_seq" in lsa.lib().lsa_last_error().decode()
    assert lsa.prefill_attn_workspace_size(F(4, 1, 64, 64, 0.1), MOST, 10, 5000) > 0
    assert lsa.prefill_attn_workspace_size(F(4, 1, 64, 64, 0.1), MOST + 1, 10, 5000) == 0
    assert lsa.chunk_attn_workspace_size(C(4, 1, 64, 64, False, 0.1), MOST, 10, 100, 64) > 0
    assert lsa.chunk_attn_workspace_size(C(4, 1, 64, 64, False, 0.1), MOST + 1, 10, 100, 64) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [MOST, 40])
def test_the_most_sequences(tokens):
    """65536 sequences of a token and two keys each, and 40 tokens of 40 of them; the second key is the token's own position."""
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=dev).to(torch.bfloat16)
    prm = F(2, 1, 64, 64, 0.125)
    q, k, v = r(tokens, 2, 64), r(2 * MOST, 1, 64), r(2 * MOST, 1, 64)
    own = torch.arange(tokens, device=dev) * (MOST // tokens) + MOST // tokens - 1      # the sequence of a token
    cu_q = torch.searchsorted(own, torch.arange(MOST + 1, device=dev)).to(torch.int32)
    cu_kv = (2 * torch.arange(MOST + 1, device=dev)).to(torch.int32)
    assert (lsa.prefill_attn_workspace_size(prm, MOST, tokens, 2 * MOST) > 0) == (tokens == 40)
    out, lse = lsa.prefill_attn(prm, q, k, v, cu_q, cu_kv)
    kk, vv = k.view(MOST, 2, 64)[own].double(), v.view(MOST, 2, 64)[own].double()
    s = (q.double()[:, :, None] * kk[:, None]).sum(-1) * 0.125                          # [tokens, 2, 2]
    p = torch.softmax(s, -1)
    want, spread = (p[..., None] * vv[:, None]).sum(2), (p[..., None] * vv.abs()[:, None]).sum(2)
    # the bound of tests/prompt_check.py for two keys: weights and output rounded to bf16, scores off by at most 66 * 2^-23 * 0.125 sum |q_i k_i| < 2^-13
    # (the sum below 120)
    assert float((q.double()[:, :, None] * kk[:, None]).abs().sum(-1).max()) < 120
    assert ((out.double() - want).abs() <= (2 * 2.0 ** -8 * (1 + 2.0 ** -8) + 2 * 2.0 ** -13 + 2.0 ** -17) * spread).all()
    assert ((lse.double() - torch.logsumexp(s, -1)).abs() <= 2.0 ** -13 + 2.0 ** -17 * (1 + lse.double().abs())).all()
