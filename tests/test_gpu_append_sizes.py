"""lsa_cache_append calls of more threads than one launch of the runtime takes (2^32)."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16


def test_an_append_of_many_threads():
    """Keys and values of 33 units a head, dealt to 64 lanes each: 2^31 threads of either in 2^25 token heads, and the
    queries' threads. Keys and values are one tensor, and all tokens but a few have no position."""
    heads, d = 128, 528
    n = (1 << 18) + 2
    prm = lsa.AppendParams(8, heads, d, d, 0, 16, False, True)
    x = torch.zeros((n, heads, d), dtype=BF, device=DEV)
    q = torch.zeros((n, 8, d), dtype=BF, device=DEV)
    some = [0, 5, n // 2, n - 3, n - 1]
    g = torch.Generator(device=DEV).manual_seed(2)
    small = torch.randn((len(some), heads, d), generator=g, device=DEV).to(BF)
    small_q = torch.randn((len(some), 8, d), generator=g, device=DEV).to(BF)
    pos = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    for i, t in enumerate(some):
        x[t], q[t] = small[i], small_q[i]
        pos[t] = i
    rope = torch.randn((8, 16), generator=g, device=DEV)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)

    def caches():
        c = lambda: torch.zeros((1, heads, 8, d), dtype=torch.uint8, device=DEV)
        s = lambda: torch.zeros((1, heads, 8), device=DEV)
        return dict(k_cache=c(), v_cache=c(), k_scale=s(), v_scale=s())
    a, b = caches(), caches()
    q_out, rows = lsa.cache_append(prm, x, q=q, page_table=table, pos=pos, seq=torch.zeros(n, dtype=torch.int32, device=DEV), rope=rope, v=x,
                               rows=True, **a)
    want, _ = lsa.cache_append(prm, small, q=small_q, page_table=table, pos=torch.arange(len(some), dtype=torch.int32, device=DEV),
                     seq=torch.zeros(len(some), dtype=torch.int32, device=DEV), rope=rope, v=small, **b)
    assert torch.equal(rows, pos.long()) and torch.equal(q_out[some], want) and q_out.count_nonzero() == want.count_nonzero()
    for name in a:
        assert torch.equal(a[name], b[name]) and a[name].count_nonzero() > 0, name
