"""Errors of the HIP runtime around the prompt-side operators: an error that an earlier call left pending is not theirs."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.test_prompt_bind import _chunk_call, _norm_call, _prefill_call, _read_call
from tests.test_serve_errors import _with_pending_error

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not os.path.exists(lsa.LIB_PATH), reason="liblsa.so not built")]


@pytest.mark.parametrize("call,make,kind", [(lsa.norm_append, _norm_call, "gqa"), (lsa.cache_read, _read_call, "fp8"), (lsa.prefill_attn, _prefill_call, "plain"),
                                            (lsa.prefill_attn, _prefill_call, "cut"), (lsa.chunk_attn, _chunk_call, "cut")])
def test_beside_a_pending_error(call, make, kind):
    torch.manual_seed(6)
    prm, a = make(kind)
    want = [t.clone() for t in call(prm, **a) if t is not None]
    got = _with_pending_error(lambda: [t for t in call(prm, **a) if t is not None])
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x, y)
