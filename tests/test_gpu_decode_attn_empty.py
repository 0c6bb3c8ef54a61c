"""lsa_decode_attn where every score of a row is -inf: o = 0 and lse = -inf, whatever its values hold."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_decode_attn import GQA, MLA, _batch, _params, _run

pytestmark = pytest.mark.gpu


NAN, INF = float("nan"), float("inf")
GROUPED = [(GQA, 16, 2, 128, False), (GQA, 16, 2, 64, True), (GQA, 64, 1, 128, False), (GQA, 40, 1, 64, True)]
LATENT = [(MLA, 64, 1, 576, False), (MLA, 20, 1, 576, False), (MLA, 128, 1, 576, False)]


@pytest.mark.parametrize("form,bad", [(f, bad) for f in GROUPED for bad in (NAN, INF, -INF)] + [(f, -INF) for f in LATENT], ids=str)
@pytest.mark.parametrize("ctx,width", [([150, 64, 97], None), ([2100, 900, 700], 70)], ids=["whole", "cut"])
@pytest.mark.parametrize("R", [1, 3])
def test_all_scores_minus_infinity(form, bad, ctx, width, R):
    """Positive queries against keys of -inf (fp8: negative codes of an infinite scale) in the first two sequences, whose
    values are no numbers or infinite (a latent row's are its key's -inf). The third keeps its bits."""
    prm = _params(*form)
    x = _batch(prm, ctx, R, 64, seed=R, width=width, slack=0)
    x["q"].abs_().add_(0.5)
    ref, ref_l = (y.clone() for y in _run(prm, x))
    pages = [p for b in range(2) for p in x["table"][b, :-(-ctx[b] // 64)].tolist()]
    if prm.fp8:
        x["k_cache"].view(torch.uint8)[pages] = torch.tensor(-1.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
        x["k_scale"][pages] = INF
        x["v_cache"].view(torch.uint8)[pages] = 0x7F if bad != bad else 0x38
        x["v_scale"][pages] = bad
    else:
        x["k_cache"][pages] = -INF
        if not prm.latent:
            x["v_cache"][pages] = bad
    out, lse = _run(prm, x)
    n = 2 * R
    assert (lse[:n] == -INF).all() and (out[:n] == 0).all()
    assert torch.equal(out[n:], ref[n:]) and torch.equal(lse[n:], ref_l[n:])
