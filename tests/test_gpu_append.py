"""lsa_cache_append against the float64 oracle: rotation of queries and keys, and their rows in the caches.

Tolerances, from the arithmetic (u = 2^-24): a rotated value a c - b s is two fp32 products and a sum, off by
at most 3 u (|a| + |b|), then rounded once to bf16 (8 significant bits: 2^-8 relative). An fp8 row: since a rotation keeps the
length of a pair, |a| + |b| <= 2 max|x'| over the row, so the scale max|x'| / 448 is off by at most 7 u
relative, and a code stands for its value within half a step of e4m3: 2^-4 relative, or 2^-10 of the scale
below the normal range. What is copied is equal."""
from __future__ import annotations

import pytest
import torch

import oracle.serve_oracle as orc
from paper_2608_01662_amd import lsa

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24


def _randn(shape, g):
    return torch.randn(shape, generator=g).to(torch.bfloat16)


def _rope(n_pos, dim):
    freq = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) / max(1, dim // 2))
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * freq
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def _setup(prm, lens, new, page, seed, split=False, fused=False):
    """A batch whose sequences hold `lens` tokens, `new` of each being appended: host tensors, with a permuted
    page table. split: the rotated parts apart; fused: q, k, v slices of one tensor."""
    g = torch.Generator().manual_seed(seed)
    n_seq = len(lens)
    pages = [-(-x // page) for x in lens]
    n_phys, width = sum(pages) + 2, max(pages + [1])
    perm = torch.randperm(n_phys, generator=g).tolist()
    table, at = [], 0
    for p in pages:
        table.append(perm[at:at + p] + [-1] * (width - p))
        at += p
    seq = [b for b in range(n_seq) for _ in range(new[b])]
    pos = [lens[b] - new[b] + j for b in range(n_seq) for j in range(new[b])]
    n = len(seq)
    H, Hk, dk, dv, rd = prm.n_heads, prm.n_kv_heads, prm.d_k, prm.d_v, prm.rot_dim
    d = {}
    if fused:
        # (wider than its parts, so that the tokens' stride is no multiple of a head)
        f = _randn((n, H * dk + Hk * dk + Hk * dv + 8), g)
        d["fused"] = f
        d["q"], d["k"] = f[:, :H * dk].unflatten(1, (H, dk)), f[:, H * dk:H * dk + Hk * dk].unflatten(1, (Hk, dk))
        if dv:
            d["v"] = f[:, H * dk + Hk * dk:-8].unflatten(1, (Hk, dv))
    else:
        cut = rd if split else 0
        if H:
            d["q"] = _randn((n, H, dk - cut), g)
        d["k"] = _randn((n, Hk, dk - cut), g)
        if split:
            d["k_rot"] = _randn((n, Hk, rd), g)
            if H:
                d["q_rot"] = _randn((n, H, rd), g)
        if dv:
            d["v"] = _randn((n, Hk, dv), g)
    rope = _rope(max(lens + [1]), rd) if rd else None
    return dict(d, seq=seq, pos=pos, table=table, n_phys=n_phys, page=page, rope=rope, lens=lens, n=n)


def _caches(prm, s, fill=7.0):
    shape = lambda d: (s["n_phys"], prm.n_kv_heads, s["page"], d)
    kind = torch.uint8 if prm.fp8 else torch.bfloat16
    c = dict(k_cache=torch.full(shape(prm.d_k), 33 if prm.fp8 else fill, dtype=kind, device=DEV))
    if prm.d_v:
        c["v_cache"] = torch.full(shape(prm.d_v), 33 if prm.fp8 else fill, dtype=kind, device=DEV)
    if prm.fp8:
        c["k_scale"] = torch.full(shape(1)[:3], fill, device=DEV)
        if prm.d_v:
            c["v_scale"] = torch.full(shape(1)[:3], fill, device=DEV)
    return c


def _dev_inputs(s):
    names = [x for x in ("q", "q_rot", "k", "k_rot", "v") if x in s]
    if "fused" in s:
        f = s["fused"].to(DEV)
        out, off = {}, 0
        for x in names:
            w = s[x].shape[1] * s[x].shape[2]
            out[x] = f[:, off:off + w].unflatten(1, tuple(s[x].shape[1:]))
            off += w
        return out
    return {x: s[x].to(DEV) for x in names}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _check(prm, s, caches, q_out, rows, rope_rows=None):
    n, page = s["n"], s["page"]
    want_rows = [orc.cache_row(b, p if not prm.rot_dim or p < rope_rows else -1, s["table"], page, len(s["lens"]), s["n_phys"])
                 for b, p in zip(s["seq"], s["pos"])]
    if rows is not None:
        assert rows.tolist() == want_rows

    def whole(x, part):
        return torch.cat([s[x], s[part]], 2).double() if part in s else s[x].double()

    def rotated(x, t):
        if not prm.rot_dim:
            return x
        return orc.rotate(x, prm.rot_start, prm.rot_dim, prm.interleaved, s["rope"][s["pos"][t]])

    def reach(x):  # bounds |a| + |b| of every pair of a head
        return 2 * x.abs().amax(-1, keepdim=True)
    if prm.n_heads:
        q, got = whole("q", "q_rot"), q_out.double().cpu()
        for t in range(n):
            valid = 0 <= s["seq"][t] < len(s["lens"]) and 0 <= s["pos"][t] < len(s["table"][0]) * page and \
                (not prm.rot_dim or s["pos"][t] < rope_rows)
            want = rotated(q[t], t) if valid else torch.zeros_like(q[t])
            tol = 1.01 * 2.0 ** -8 * want.abs() + 3 * U * reach(q[t])
            if not prm.rot_dim:
                tol = tol * 0
            assert ((got[t] - want).abs() <= tol).all(), t
    for x, d in (("k", prm.d_k), ("v", prm.d_v)):
        if not d:
            continue
        src = whole("k", "k_rot") if x == "k" else s["v"].double()
        cache = caches[x + "_cache"]
        flat = cache.transpose(1, 2).reshape(-1, prm.n_kv_heads, d).cpu()      # [rows, heads, d]
        scales = caches[x + "_scale"].transpose(1, 2).reshape(-1, prm.n_kv_heads).cpu() if prm.fp8 else None
        written = torch.zeros(flat.shape[0], dtype=torch.bool)
        for t, r in enumerate(want_rows):
            if r < 0:
                continue
            written[r] = True
            want = rotated(src[t], t) if x == "k" else src[t]
            if not prm.fp8:
                tol = 1.01 * 2.0 ** -8 * want.abs() + 3 * U * reach(src[t])
                if x == "v" or not prm.rot_dim:
                    tol = tol * 0
                assert ((flat[r].double() - want).abs() <= tol).all(), (x, t)
                continue
            top = want.abs().amax(1)
            ws = torch.where(top > 0, (top / 448).clamp_min(2.0 ** -126), torch.ones_like(top))
            assert ((scales[r].double() - ws).abs() <= 7 * U * ws).all(), (x, t)
            got = flat[r].view(torch.float8_e4m3fn).double() * scales[r].double()[:, None]
            tol = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * ws[:, None]) * (1 + 2.0 ** -10) + 8 * U * reach(src[t])
            assert ((got - want).abs() <= tol).all(), (x, t)
        # what was not written is as it was
        rest = flat[~written]
        assert (rest == (33 if prm.fp8 else 7.0)).all(), x
        if prm.fp8:
            assert (scales[~written] == 7.0).all(), x


A = lsa.AppendParams
FORMS = [
    # grouped heads, both pairings, whole and partial rotation, one and many key heads
    (A(8, 2, 128, 128, 0, 128, False, False), dict(fused=True)),
    (A(8, 2, 128, 128, 0, 64, True, True), dict(fused=True)),
    (A(5, 5, 64, 64, 0, 64, False, True), {}),
    (A(16, 1, 128, 128, 32, 96, True, False), dict(fused=True)),
    (A(3, 1, 80, 48, 16, 32, False, True), {}),           # widths that are no power of two
    (A(4, 2, 16, 1024, 0, 16, False, True), {}),          # the least and the greatest width
    (A(2, 1, 1024, 16, 0, 1024, True, True), {}),
    (A(4, 2, 64, 64), dict(fused=True)),                  # no rotation: copies
    (A(0, 3, 64, 64, 0, 32, False, False), {}),           # no queries
    # latent row from its parts, and whole
    (A(64, 1, 576, 0, 512, 64, True, False), dict(split=True)),
    (A(16, 1, 576, 0, 512, 64, False, False), dict(split=True)),
    (A(2, 1, 576, 0, 512, 64, True, True), {}),
    # indexer keys
    (A(32, 1, 128, 0, 0, 64, True, True), {}),
    (A(8, 1, 64, 0, 0, 64, True, False), dict(fused=True)),
]


@pytest.mark.parametrize("prm,kw", FORMS, ids=lambda x: "-".join(str(v) for v in vars(x).values()) if hasattr(x, "d_k") else "")
@pytest.mark.parametrize("page", [64, 37, 1])
def test_append_forms(prm, kw, page):
    """Every form, tokens of a ragged batch by sequence and position, pages of 64, 37 and one token."""
    s = _setup(prm, [1, 70, 5, 131], [1, 3, 5, 31], page, seed=page, **kw)
    c, x = _caches(prm, s), _dev_inputs(s)
    q, rows = lsa.cache_append(prm, x.pop("k"), c["k_cache"], page_table=_i32(s["table"]), pos=_i32(s["pos"]),
                               seq=_i32(s["seq"]), rope=None if s["rope"] is None else s["rope"].to(DEV), rows=True,
                               **x, **{k: v for k, v in c.items() if k != "k_cache"})
    _check(prm, s, c, q, rows, len(s["rope"]) if s["rope"] is not None else None)


@pytest.mark.parametrize("new", [1, 3])
def test_append_by_context_length(new):
    """The decode form: the last tokens of each sequence, by its length; equal to the same by position."""
    prm = A(8, 2, 128, 128, 0, 128, False, True)
    s = _setup(prm, [new, 40, 64, 65, 500], [new] * 5, 64, seed=new)
    x, rope, table = _dev_inputs(s), s["rope"].to(DEV), _i32(s["table"])
    a, b = _caches(prm, s), _caches(prm, s)
    k = x.pop("k")
    qa, ra = lsa.cache_append(prm, k, page_table=table, ctx_len=_i32(s["lens"]), rows_per_seq=new, rope=rope, rows=True, **x, **a)
    qb, rb = lsa.cache_append(prm, k, page_table=table, pos=_i32(s["pos"]), rows_per_seq=new, rope=rope, rows=True, **x, **b)
    _check(prm, s, a, qa, ra, len(rope))
    assert torch.equal(qa, qb) and torch.equal(ra, rb)
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_append_skips_what_has_no_row():
    """Sequences and positions out of range, unmapped pages and positions beyond the angle table: nothing is
    cached, rows are -1; queries of tokens without a position are zeros, others rotated."""
    prm = A(2, 2, 64, 64, 0, 64, False, False)
    s = _setup(prm, [100, 100, 100], [4, 4, 4], 16, seed=9)
    s["seq"][0], s["seq"][1], s["pos"][2] = -1, 3, -1
    s["pos"][3] = len(s["table"][0]) * 16          # beyond the table
    s["table"][1][s["pos"][4] // 16] = s["n_phys"]  # outside the pool
    s["table"][2][s["pos"][8] // 16] = -5
    s["pos"][5] = 2 ** 31 - 1
    s["rope"] = s["rope"][:99]                      # the last position of each has no angles
    c, x = _caches(prm, s), _dev_inputs(s)
    q, rows = lsa.cache_append(prm, x.pop("k"), page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                               rope=s["rope"].to(DEV), rows=True, **x, **c)
    assert (rows == -1).sum() >= 7
    _check(prm, s, c, q, rows, 99)
    # an idle slot of a decode batch (length 0) and one shorter than the new tokens
    s = _setup(prm, [3, 50, 64], [3, 3, 3], 16, seed=3)
    lens = [0, 2, 64]
    s["pos"] = [l - 3 + j for l in lens for j in range(3)]
    c, x = _caches(prm, s), _dev_inputs(s)
    q, rows = lsa.cache_append(prm, x.pop("k"), page_table=_i32(s["table"]), ctx_len=_i32(lens), rows_per_seq=3,
                               rope=s["rope"].to(DEV), rows=True, **x, **c)
    assert rows[:4].tolist() == [-1] * 4 and (rows[4:] >= 0).all()
    _check(prm, s, c, q, rows, len(s["rope"]))


def test_append_without_page_table_and_in_place():
    """Contiguous caches (a page per sequence), queries rotated where they are; no heads dimension."""
    prm = A(6, 1, 64, 64, 0, 64, False, False)
    s = _setup(prm, [9, 33, 40], [9, 33, 40], 40, seed=4)
    s["table"], s["n_phys"] = [[0], [1], [2]], 3
    c, x = _caches(prm, s), _dev_inputs(s)
    q0 = x.pop("q")
    q, rows = lsa.cache_append(prm, x["k"], c["k_cache"][:, 0], pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                               rope=s["rope"].to(DEV), v=x["v"], v_cache=c["v_cache"][:, 0], q=q0, q_out=q0, rows=True)
    assert q is q0
    _check(prm, s, c, q, rows, len(s["rope"]))


def test_append_fp8_of_zeros_tiny_and_non_finite_rows():
    """A zero row has scale 1; a row whose largest value over 448 leaves the normal range keeps the least normal
    scale; a NaN or an infinity is not hidden: the row's scale or codes are not finite, other rows unharmed."""
    prm = A(0, 1, 64, 64, fp8=True)
    s = _setup(prm, [5], [5], 16, seed=2)
    s["k"][0] = 0
    s["k"][1] = 1e-39
    s["k"][2, 0, 5], s["k"][3, 0, 63] = float("nan"), float("inf")
    c = _caches(prm, s)
    _, rows = lsa.cache_append(prm, s["k"].to(DEV), page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                               v=s["v"].to(DEV), rows=True, **c)
    codes = c["k_cache"].view(torch.float8_e4m3fn).float().reshape(-1, 64)[rows].cpu()
    scale = c["k_scale"].reshape(-1)[rows].cpu()
    assert scale[0] == 1 and (codes[0] == 0).all()
    assert scale[1] == 2.0 ** -126
    deq = codes * scale[:, None]
    assert ((deq[1] - s["k"][1, 0].float()).abs() <= 2.0 ** -4 * 1e-39 * 1.01).all()
    assert not torch.isfinite(deq[2]).any() and not torch.isfinite(deq[3]).any()
    want = s["k"][4, 0].float()
    assert ((deq[4] - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * scale[4]) * 1.001).all()
    vals = (c["v_cache"].view(torch.float8_e4m3fn).float() * c["v_scale"][..., None]).reshape(-1, 64)[rows].cpu()
    assert torch.isfinite(vals).all()


def test_append_rows_feed_the_block_cache_and_large_offsets():
    """`rows` goes to block_keys_update as it is; rows of a cache past 2^31 elements and 2^32 bytes."""
    page, n_phys = 64, (1 << 32) // (64 * 576 * 2) + 20
    prm = A(0, 1, 576, 0, 512, 64, True, False)
    s = _setup(prm, [200, 3], [200, 3], page, seed=8)
    top = [n_phys - 1, n_phys - 3, 0, n_phys // 2]
    s["table"] = [top, [n_phys - 2, -1, -1, -1]]
    cache = torch.zeros((n_phys, page, 576), dtype=torch.bfloat16, device=DEV)
    _, rows = lsa.cache_append(prm, s["k"].to(DEV), cache, page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                               rope=s["rope"].to(DEV), rows=True)
    want = [orc.cache_row(b, p, s["table"], page, 2, n_phys) for b, p in zip(s["seq"], s["pos"])]
    assert rows.tolist() == want and max(want) * 576 > 1 << 31
    got = cache.view(-1, 576)[rows].double().cpu()
    for t in (0, 63, 64, 128, 199, 200, 202):
        ref = orc.rotate(s["k"][t].double(), 512, 64, True, s["rope"][s["pos"][t]])[0]
        assert ((got[t] - ref).abs() <= 1.01 * 2.0 ** -8 * ref.abs() + 6 * U * ref.abs().max()).all()
    assert int((cache != 0).any(-1).sum()) == len(set(want))
    del cache
    # block cache of fp8 indexer keys, kept current through the rows
    ip = lsa.IndexParams(8, 64, True, 64, 32, 4, 64, 4, 64, 64)
    prm = A(8, 1, 64, 0, 0, 64, True, True)
    s = _setup(prm, [64, 100], [64, 100], page, seed=5)
    x, c = _dev_inputs(s), _caches(prm, s)
    _, rows = lsa.cache_append(prm, x["k"], page_table=_i32(s["table"]), pos=_i32(s["pos"]), seq=_i32(s["seq"]),
                               rope=s["rope"].to(DEV), q=x["q"], rows=True, **c)
    keys, scales = c["k_cache"].view(-1, 64), c["k_scale"].view(-1)
    block = lsa.block_keys(ip, keys, scales)
    stale = torch.zeros_like(block)
    lsa.block_keys_update(ip, rows, keys, scales, stale)
    hit = torch.unique(rows // 32)
    assert torch.equal(stale[hit], block[hit])


def test_append_refusals():
    prm = A(4, 2, 64, 64, 0, 64, False, False)
    n, dev = 3, DEV
    x = dict(k=torch.zeros((n, 2, 64), dtype=torch.bfloat16, device=dev), v=torch.zeros((n, 2, 64), dtype=torch.bfloat16, device=dev),
             q=torch.zeros((n, 4, 64), dtype=torch.bfloat16, device=dev), k_cache=torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device=dev),
             v_cache=torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device=dev), rope=torch.zeros((64, 64), device=dev),
             page_table=torch.zeros((3, 1), dtype=torch.int32, device=dev), ctx_len=torch.ones(3, dtype=torch.int32, device=dev))
    call = lambda p=prm, **kw: lsa.cache_append(p, **{**x, **kw})
    wide = torch.zeros((n, 2, 128), dtype=torch.bfloat16, device=dev)
    for kw, word in [
        (dict(k=wide[..., :64]), "contiguous"), (dict(k=x["k"].float()), "dtype"), (dict(v=None), "v must"),
        (dict(q=x["q"][:2]), "shape"), (dict(k=x["k"].cpu()), "CUDA"), (dict(v_cache=x["v_cache"][:3]), "pages"),
        (dict(k_scale=torch.zeros((4, 2, 16), device=dev)), "None"), (dict(rope=x["rope"][:, :32].contiguous()), "shape"),
        (dict(pos=x["ctx_len"]), "exactly one"), (dict(ctx_len=None), "exactly one"), (dict(rows_per_seq=2), "tokens"),
        (dict(seq=x["ctx_len"]), "seq must"), (dict(rows=x["ctx_len"]), "dtype"), (dict(n_seq=2), "n_seq"),
        (dict(rope=None), "rope"),
    ]:
        with pytest.raises(ValueError, match=word):
            call(**kw)
    flat = torch.zeros(n * 128 + 4, dtype=torch.bfloat16, device=dev)
    with pytest.raises(lsa.LSAError, match="aligned"):
        call(k=flat[4:4 + n * 128].view(n, 2, 64))
    with pytest.raises(lsa.LSAError, match="multiples of 16"):
        call(A(4, 2, 64, 64, 0, 24), rope=torch.zeros((64, 24), device=dev))
    with pytest.raises(lsa.LSAError, match="k_rot"):            # the rotated dims are not the last
        call(A(4, 2, 64, 64, 0, 32), k=torch.zeros((n, 2, 32), dtype=torch.bfloat16, device=dev), rope=x["rope"][:, :32].contiguous(),
             k_rot=torch.zeros((n, 2, 32), dtype=torch.bfloat16, device=dev))


@pytest.mark.parametrize("prm,kw,n", [(A(32, 8, 128, 128, 0, 64, False, True), dict(fused=True), 2100),
                                      (A(64, 1, 576, 0, 512, 64, True, False), dict(split=True), 300),
                                      (A(36, 4, 64, 64, 16, 32, True, False), {}, 4000)], ids=["gqa", "latent", "partial"])
def test_large_calls_equal_small_ones(prm, kw, n):
    """A call of many tokens (several query heads per thread) gives the bits of the same tokens in small calls."""
    s = _setup(prm, [n // 3 + 40, n - n // 3 + 5], [n // 3, n - n // 3], 64, seed=n, **kw)
    x, rope, table = _dev_inputs(s), s["rope"].to(DEV), _i32(s["table"])
    pos, seq = _i32(s["pos"]), _i32(s["seq"])
    seq[5] = 7      # no such sequence: zero queries in both
    a, b = _caches(prm, s), _caches(prm, s)
    q, rows = lsa.cache_append(prm, page_table=table, pos=pos, seq=seq, rope=rope, rows=True, **x, **a)
    for t in range(0, n, 97):
        part = slice(t, min(n, t + 97))
        qs, rs = lsa.cache_append(prm, page_table=table, pos=pos[part], seq=seq[part], rope=rope, rows=True,
                                  **{k: v[part] for k, v in x.items()}, **b)
        assert torch.equal(qs, q[part]) and torch.equal(rs, rows[part])
    for name in a:
        assert torch.equal(a[name], b[name]), name
