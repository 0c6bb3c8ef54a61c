"""lsa_cache_read: packed rows of a paged cache. What is bf16 comes back equal; of fp8 caches a value is one fp32 product
(2^-24 relative) rounded once to bf16: equal to the fp32 product rounded by torch."""
from __future__ import annotations

import pytest
import torch

from paper_2608_01662_amd import lsa

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
R = lsa.CacheReadParams


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cache(n_phys, heads, page, d, fp8, g):
    if fp8:
        codes = torch.randint(0, 256, (n_phys, heads, page, d), generator=g).to(torch.uint8)
        codes[(codes & 0x7F) == 0x7F] = 0x38                     # no NaN
        return codes, torch.rand((n_phys, heads, page), generator=g) * 3
    return torch.randn((n_phys, heads, page, d), generator=g).to(torch.bfloat16), None


def _row(cache, scale, table, b, pos, page):
    """Row [heads, d] of a position, zeros without one."""
    if pos < 0 or pos // page >= len(table[b]) or not 0 <= table[b][pos // page] < cache.shape[0]:
        return torch.zeros((cache.shape[1], cache.shape[3]), dtype=torch.bfloat16)
    at = table[b][pos // page], slice(None), pos % page
    if scale is None:
        return cache[at]
    return (cache[at].view(torch.float8_e4m3fn).float() * scale[at][:, None]).to(torch.bfloat16)


def _run(prm, page, lens, start=None, n_tok=None, lead=0, bad=(), seed=0, mapped=None):
    """Sequences of `lens` rows from `start` on, `lead` rows of the output before the first; `bad`: (sequence, page) unmapped."""
    g = torch.Generator().manual_seed(seed)
    begin = start or [0] * len(lens)
    pages = [max(1, -(-(s + n) // page)) for s, n in zip(begin, lens)] if mapped is None else [mapped] * len(lens)
    n_phys = sum(pages) + 3
    perm = torch.randperm(n_phys, generator=g).tolist()
    table, at = [], 0
    for p in pages:
        table.append(perm[at:at + p] + [-1] * (max(pages) - p))
        at += p
    for i, (b, p) in enumerate(bad):
        table[b][p] = [-1, n_phys, -2 ** 31][i % 3]
    k, ks = _cache(n_phys, prm.n_kv_heads, page, prm.d_k, prm.fp8, g)
    v, vs = _cache(n_phys, prm.n_kv_heads, page, prm.d_v, prm.fp8, g) if prm.d_v else (None, None)
    cu = [lead]
    for n in lens:
        cu.append(cu[-1] + n)
    n_tok = cu[-1] if n_tok is None else n_tok
    to = lambda t: None if t is None else t.to(DEV)
    out = {x: torch.full((n_tok, prm.n_kv_heads, d), 7.0, dtype=torch.bfloat16, device=DEV) for x, d in (("k_out", prm.d_k), ("v_out", prm.d_v)) if d}
    got = lsa.cache_read(prm, to(k), _i32(cu), n_tok, page_table=_i32(table), start=None if start is None else _i32(start), v_cache=to(v),
                         k_scale=to(ks), v_scale=to(vs), **out)
    for c, s, o in ((k, ks, got[0]), (v, vs, got[1])):
        if c is None:
            assert o is None
            continue
        want = torch.full(o.shape, 7.0, dtype=torch.bfloat16)
        for b, n in enumerate(lens):
            for i in range(n):
                if cu[b] + i < n_tok:
                    want[cu[b] + i] = _row(c, s, table, b, begin[b] + i, page)
        assert torch.equal(o.cpu(), want)


FORMS = [R(8, 128, 128), R(8, 128, 128, True), R(1, 576), R(1, 576, 0, True), R(3, 80, 48, True), R(2, 16, 1024), R(5, 64, 64)]


@pytest.mark.parametrize("prm", FORMS, ids=str)
@pytest.mark.parametrize("page", [64, 20, 1])
def test_forms(prm, page):
    _run(prm, page, [1, 0, 70, 5, 131, 0], seed=page)


@pytest.mark.parametrize("fp8", [False, True])
def test_starts_leads_and_rows_behind(fp8):
    """Rows from the middle of sequences; rows of the output before the first and behind the last sequence, which stay as they were;
    an output that ends inside a sequence; positions beyond the table and before 0, unmapped pages."""
    prm = R(2, 64, 32, fp8)
    _run(prm, 16, [40, 3, 0, 17], start=[5, 100, 7, 16], lead=2, n_tok=70)
    _run(prm, 16, [40, 30], n_tok=55)
    _run(prm, 16, [40, 30, 20], start=[30, -7, 2 ** 31 - 4], mapped=4)
    _run(prm, 16, [64, 64], bad=[(0, 1), (1, 0), (1, 3)])


@pytest.mark.parametrize("n_seq,least,most", [(300, 0, 9), (1, 5000, 5000), (3, 1, 3000)])
def test_many_sequences_and_long_ones(n_seq, least, most):
    """More rows than one workgroup takes, sequences that end within one."""
    lens = torch.randint(least, most + 1, (n_seq,), generator=torch.Generator().manual_seed(n_seq)).tolist()
    _run(R(1, 16, 16, n_seq == 3), 64, lens)


def test_without_a_table_and_one_head():
    """Sequence b has page b alone; caches of one head without the head dimension; outputs made by the call."""
    g = torch.Generator().manual_seed(1)
    cache = torch.randn((4, 32, 64), generator=g).to(torch.bfloat16)
    k, v = lsa.cache_read(R(1, 64), cache.to(DEV), _i32([0, 32, 37, 37]), 37)
    assert v is None and torch.equal(k[:, 0].cpu(), torch.cat([cache[0], cache[1, :5]]))
    k, _ = lsa.cache_read(R(1, 64), cache.to(DEV), _i32([0]), 5)
    assert k.shape == (5, 1, 64)
    k, _ = lsa.cache_read(R(1, 64), cache.to(DEV), _i32([0, 0]), 0)
    assert k.shape == (0, 1, 64)


def test_reads_what_was_appended():
    """norm_append's keys beside the cache and what is read back are the same rows."""
    prm = lsa.AppendParams(2, 2, 64, 64, 0, 64, False, False)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((50, 2, 64), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    kc, vc = (torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = _i32([[3, 0, -1], [5, 1, 2]])
    seq, pos = _i32([0] * 20 + [1] * 30), _i32(list(range(20)) + list(range(10, 40)))
    rope = torch.randn((48, 64), generator=g).to(DEV)
    _, keys, _ = lsa.norm_append(prm, k, kc, v=v, v_cache=vc, q=k, k_weight=k[0, 0].contiguous(), k_out=True, page_table=table, seq=seq, pos=pos, rope=rope)
    a, b = lsa.cache_read(R(2, 64, 64), kc, _i32([0, 20, 50]), 50, v_cache=vc, page_table=table, start=_i32([0, 10]))
    assert torch.equal(a, keys) and torch.equal(b, v)


def test_in_a_graph():
    """Captured once, replayed over other offsets and contents."""
    g = torch.Generator().manual_seed(3)
    cache = torch.zeros((8, 2, 16, 32), dtype=torch.bfloat16, device=DEV)
    cu, table = _i32([0, 0, 0]), _i32([[0, 1, 2, 3], [7, 6, 5, 4]])
    prm = R(2, 32)
    lsa.cache_read(prm, cache, cu, 100, page_table=table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    out = torch.zeros((100, 2, 32), dtype=torch.bfloat16, device=DEV)
    with torch.cuda.graph(graph):
        lsa.cache_read(prm, cache, cu, 100, page_table=table, k_out=out)
    for a, b in ((10, 60), (0, 64), (50, 100)):
        cache.copy_(torch.randn(cache.shape, generator=g).to(torch.bfloat16))
        cu.copy_(torch.tensor([0, a, b], dtype=torch.int32))
        graph.replay()
        want = lsa.cache_read(prm, cache, cu, 100, page_table=table)[0]
        torch.cuda.synchronize()
        assert torch.equal(out[:b], want[:b])
