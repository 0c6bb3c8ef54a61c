"""Measured cases of the serving operators for prompts: normalising and rotating new queries and keys on their way into a
paged cache, reading a cache back into packed rows, attention over packed prompts, and attention of ragged chunks of new
tokens over a paged cache.

A case names one call and its sizes. Lengths follow from the case alone (`mix` picks how a total is dealt to the
sequences), so that its work is known. Sizes come from the package's presets (64 heads of a 512 + 64 latent cache whose
unabsorbed heads are 192 / 128 wide, 16 x 128 MQA, 64-token pages, 16K to 128K contexts, chunks of 8192) or are the
ordinary grouped-head ones.
"""
import random

import torch

own = False     # False: the plain form of the operators; True: the package's entry points

DEV = "cuda"
FP8 = torch.float8_e4m3fn
LATENT, ROT = 512, 64
EPS = 1e-6


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one interactive user of a grouped-head layer with normed queries and keys: one token, latency
        dict(name="norm_append_b1", op="norm_append", kind="gqa", heads=32, kv_heads=8, d=128, fp8=False, page=64, rot_dim=128,
             interleaved=False, n_seq=1, new=1, ctx=4096, decode=True, keys=False, mix=1),
        # the 64-sequence decode preset: the latent is normed, its rotated part and the absorbed queries only turned
        dict(name="norm_append_latent_b64", op="norm_append", kind="latent", heads=64, kv_heads=1, d=LATENT + ROT, fp8=False,
             page=64, rot_dim=ROT, interleaved=True, n_seq=64, new=64, ctx=4096, decode=True, keys=False, mix=2),
        # a chunk of the long-prompt preset's size into an fp8 cache, its keys also kept for the prompt's own attention
        dict(name="norm_append_fp8_chunk8192", op="norm_append", kind="gqa", heads=32, kv_heads=8, d=128, fp8=True, page=64,
             rot_dim=64, interleaved=False, n_seq=3, new=8192, ctx=4096, decode=False, keys=True, mix=3),
        # a short chat read back from an fp8 cache
        dict(name="cache_read_fp8_b1_1001", op="cache_read", kind="gqa", kv_heads=8, d=128, fp8=True, page=64, n_seq=1,
             ctx=1001, mix=1),
        # the latent rows of four long contexts, before their up-projection
        dict(name="cache_read_latent_128k", op="cache_read", kind="latent", kv_heads=1, d=LATENT + ROT, fp8=False, page=64,
             n_seq=4, ctx=131072, mix=2),
        # one short question to the MQA model: latency
        dict(name="prefill_mqa_129", op="prefill", heads=16, kv_heads=1, d_qk=128, d_v=128, n_seq=1, new=129, past=0,
             causal=True, k_sink=0, k_swa=0, mix=1),
        # prompts of several users packed in one call, grouped heads
        dict(name="prefill_gqa_packed16001", op="prefill", heads=32, kv_heads=8, d_qk=128, d_v=128, n_seq=7, new=16001, past=0,
             causal=True, k_sink=0, k_swa=0, mix=2),
        # the latent model's unabsorbed heads: a chunk of two prompts behind rows that were read back
        dict(name="prefill_mla_4096_past12k", op="prefill", heads=64, kv_heads=64, d_qk=192, d_v=128, n_seq=2, new=4096,
             past=12288, causal=True, k_sink=0, k_swa=0, mix=3),
        # a layer of sink and sliding window, a key per query head, 64 wide
        dict(name="prefill_swa_d64_8192", op="prefill", heads=12, kv_heads=12, d_qk=64, d_v=64, n_seq=1, new=8192, past=0,
             causal=True, k_sink=4, k_swa=1024, mix=1),
        # the last few tokens of one long document in an fp8 cache: few rows, a long axis
        dict(name="chunk_fp8_b1_16_32k", op="chunk", heads=32, kv_heads=8, d=128, fp8=True, page=64, n_seq=1, new=16,
             past=32768, k_sink=0, k_swa=0, mix=1),
        # a server's step: chunks of some prompts beside the single tokens of others
        dict(name="chunk_mixed_b24", op="chunk", heads=32, kv_heads=8, d=128, fp8=False, page=64, n_seq=24, new=2048,
             past=98304, k_sink=0, k_swa=0, mix=5),
        # one chunk of a long prompt, the preset's 8192 rows, behind 56K cached tokens in fp8; the largest call
        dict(name="chunk_fp8_8192_64k", op="chunk", heads=32, kv_heads=8, d=128, fp8=True, page=64, n_seq=1, new=8192,
             past=57344, k_sink=0, k_swa=0, mix=1),
    ]


def _log_int(rng, lo, hi):
    """Log-uniform whole number in [lo, hi]; every other one odd."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.5:
        v |= 1
    return max(lo, min(hi, v))


_HEADS = [(32, 8), (32, 8), (16, 1), (8, 8), (28, 4), (40, 5), (64, 8), (12, 12), (16, 2)]
_PAGES = [16, 64, 64, 128, 256, 100, 37]


def _draw_one(rng, op):
    n_seq, mix = _log_int(rng, 1, 64), rng.randrange(1 << 30)
    heads, kv = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    window = dict(k_sink=0, k_swa=0)
    if rng.random() < 0.2:
        window = dict(k_sink=rng.choice([0, 4, 100]), k_swa=_log_int(rng, 64, 4096))
    if op == "norm_append":
        decode = rng.random() < 0.4
        c = dict(op=op, kind="gqa", heads=heads, kv_heads=kv, d=d, fp8=rng.random() < 0.5, page=rng.choice(_PAGES),
                 rot_dim=rng.choice([d, d, d // 2, 32]), interleaved=rng.random() < 0.5, n_seq=n_seq,
                 new=n_seq if decode else _log_int(rng, n_seq, 8192), ctx=_log_int(rng, 16, 4096), decode=decode,
                 keys=rng.random() < 0.5, mix=mix)
        if rng.random() < 0.3:
            c.update(kind="latent", heads=rng.choice([64, 64, 16]), kv_heads=1, d=LATENT + ROT, fp8=False, rot_dim=ROT, keys=False)
        return c
    if op == "cache_read":
        latent = rng.random() < 0.4
        return dict(op=op, kind="latent" if latent else "gqa", kv_heads=1 if latent else kv, d=LATENT + ROT if latent else d,
                    fp8=rng.random() < 0.5, page=rng.choice(_PAGES), n_seq=n_seq, ctx=_log_int(rng, n_seq, 131072), mix=mix)
    past = rng.choice([0, 1, 1]) * _log_int(rng, 16, 65536)
    if op == "prefill":
        d_qk, d_v = (d, d)
        if rng.random() < 0.3:
            heads, kv, d_qk, d_v = rng.choice([(64, 64), (32, 32), (16, 16)]) + (192, 128)
        n_seq, past, causal = min(n_seq, 16), past // 4 * rng.choice([0, 1]), rng.random() < 0.85
        return dict(op=op, heads=heads, kv_heads=kv, d_qk=d_qk, d_v=d_v, n_seq=n_seq, new=_log_int(rng, n_seq, 16384), past=past,
                    causal=causal, mix=mix, **(window if causal else dict(k_sink=0, k_swa=0)))
    return dict(op=op, heads=heads, kv_heads=kv, d=d, fp8=rng.random() < 0.5, page=rng.choice(_PAGES), n_seq=n_seq,
                new=_log_int(rng, n_seq, 8192), past=past, mix=mix, **window)


def draw(rng):
    op = rng.choice(["norm_append", "cache_read", "prefill", "prefill", "chunk", "chunk"])
    most = [max(work(c)[x] for c in listed() if c["op"] == op) for x in ("bytes", "flops")]
    while True:
        c = _draw_one(rng, op)
        whole = work({**c, "k_swa": 0}) if "k_swa" in c else work(c)    # (a window does not shorten the plain form)
        if whole["bytes"] <= most[0] and whole["flops"] <= most[1]:
            return c


# ------------------------------------------------------------------------------------------ lengths
def _deal(total, parts, rng, spread, least=0):
    """`total` in `parts` whole numbers of at least `least`, their sizes spread over a factor of e^spread."""
    w = [2.718281828 ** (spread * rng.random()) for _ in range(parts)]
    free = total - least * parts
    cuts, at = [], 0.0
    for x in w:
        at += x
        cuts.append(round(free * at / sum(w)))
    return [least + b - a for a, b in zip([0] + cuts[:-1], cuts)]


def _lengths(case):
    """(tokens before the call, new tokens) of each sequence."""
    rng, n = random.Random(case["mix"]), case["n_seq"]
    if case["op"] == "cache_read":
        return [0] * n, _deal(case["ctx"], n, rng, 2.0)
    if case["op"] == "norm_append":
        new = [1] * n if case["decode"] else _deal(case["new"], n, rng, 1.5, 1)
        return [rng.randint(0, case["ctx"]) for _ in range(n)], new
    new = _deal(case["new"], n, rng, 8.0 if case["op"] == "chunk" else 1.5, 1)
    return _deal(case["past"], n, rng, 2.0), new


def _offsets(lengths):
    at = [0]
    for x in lengths:
        at.append(at[-1] + x)
    return at


# ------------------------------------------------------------------------------------------ inputs
def _generator(seed, which, device=DEV):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 1000003 + which * 7919) & 0x7FFFFFFF)
    return g


def _normal(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).mul_(scale)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rope_table(n_pos, rot_dim):
    """[n_pos, rot_dim] fp32: rot_dim / 2 cosines, then as many sines, of the usual geometric frequencies."""
    freq = 10000.0 ** (-torch.arange(rot_dim // 2, dtype=torch.float64, device=DEV) / (rot_dim // 2))
    angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).to(torch.float32)


def _table(lengths, page, g):
    """Page table [n_seq, widest] of sequences of these lengths, pages anywhere in the pool, -1 padded, and the pool's size."""
    pages = torch.tensor([-(-n // page) for n in lengths])
    n_phys, width = max(1, int(pages.sum())), max(1, int(pages.max()))
    table = torch.full((len(pages), width), -1, dtype=torch.int64)
    table[torch.arange(width)[None] < pages[:, None]] = torch.randperm(n_phys, generator=g)[:int(pages.sum())]
    return table.to(torch.int32).to(DEV), n_phys


def _quantised(x):
    """fp8 codes and one scale per last-dimension row."""
    x = x.float()
    top = x.abs().amax(-1)
    scale = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    return (x / scale[..., None]).clamp_(-448.0, 448.0).to(FP8), scale


def prepare(case, seed):
    before, new = _lengths(case)
    at, n = _offsets(new), sum(new)
    g = _generator(seed, 3)
    st = dict(case=case, before=before, new=new, at=at, cu=_ints(at))
    ctx = [a + b for a, b in zip(before, new)]
    if case["op"] == "prefill":
        H, Hkv = case["heads"], case["kv_heads"]
        kv_at = _offsets(ctx)
        # (scores of a standard deviation near 2: some positions stand out, as in a trained layer)
        st.update(kv_at=kv_at, cu_kv=_ints(kv_at), q=_normal((n, H, case["d_qk"]), g, 2.0),
                  k=_normal((kv_at[-1], Hkv, case["d_qk"]), g), v=_normal((kv_at[-1], Hkv, case["d_v"]), g))
        return st
    Hkv, d, page = case["kv_heads"], case["d"], case["page"]
    latent = case.get("kind") == "latent"
    st["table"], n_phys = _table(ctx, page, _generator(seed, 2, "cpu"))
    st.update(ctx=_ints(ctx), ctx_list=ctx)
    shape = (n_phys, Hkv, page, d)
    if case["op"] == "norm_append":
        seq = torch.repeat_interleave(torch.arange(case["n_seq"]), torch.tensor(new))
        pos = torch.arange(n) - torch.tensor(at)[seq] + torch.tensor(before)[seq]
        st.update(seq=seq.to(torch.int32).to(DEV), pos=pos.to(torch.int32).to(DEV), rope=_rope_table(max(ctx), case["rot_dim"]))
        H = case["heads"]
        if latent:      # absorbed queries and the latent come apart from their rotated parts
            st.update(q=_normal((n, H, LATENT), g), q_rot=_normal((n, H, ROT), g), k=_normal((n, 1, LATENT), g, 3.0),
                      k_rot=_normal((n, LATENT + ROT), g)[:, LATENT:].unflatten(1, (1, ROT)),
                      k_weight=_normal((LATENT,), g, 0.2).add_(1.0))
        else:           # slices of one fused projection
            fused = _normal((n, (H + 2 * Hkv) * d), g, 3.0)
            st.update(q=fused[:, :H * d].unflatten(1, (H, d)), k=fused[:, H * d:(H + Hkv) * d].unflatten(1, (Hkv, d)),
                      v=fused[:, (H + Hkv) * d:].unflatten(1, (Hkv, d)), q_weight=_normal((d,), g, 0.2).add_(1.0),
                      k_weight=_normal((d,), g, 0.2).add_(1.0))
        for x in ["k"] if latent else ["k", "v"]:
            if case["fp8"]:
                st[x + "_cache"] = torch.zeros(shape, dtype=torch.uint8, device=DEV).view(FP8)
                st[x + "_scale"] = torch.zeros(shape[:3], dtype=torch.float32, device=DEV)
            else:
                st[x + "_cache"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        return st
    for x in ["k"] if latent else ["k", "v"]:
        st[x + "_cache"] = _normal(shape, g)
        if case["fp8"]:
            st[x + "_cache"], st[x + "_scale"] = _quantised(st[x + "_cache"])
    if case["op"] == "chunk":
        st["q"] = _normal((n, case["heads"], d), g, 2.0)
    return st


# ------------------------------------------------------------------------------------------ one pass, plain
def _rotated(x, rope, pos, interleaved):
    """x [n, heads, rot_dim] fp32 rotated by the angles of its positions."""
    half = x.shape[-1] // 2
    cos, sin = rope[pos.long()][:, None, :half], rope[pos.long()][:, None, half:]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)


def _normed_rotated(st, x, part, weight):
    """The heads in fp32, normed where there is a weight, with their rotated dims (the first, or those given apart) rotated."""
    case = st["case"]
    rot, inter = case["rot_dim"], case["interleaved"]
    x = x.float()
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.float()
    if part is not None:
        return torch.cat([x, _rotated(part.float(), st["rope"], st["pos"], inter)], dim=-1)
    return torch.cat([_rotated(x[..., :rot], st["rope"], st["pos"], inter), x[..., rot:]], dim=-1)


def _plain_norm_append(st):
    case, page = st["case"], st["case"]["page"]
    pos = st["pos"].long()
    phys, off = st["table"][st["seq"].long(), pos // page].long(), pos % page
    k = _normed_rotated(st, st["k"], st.get("k_rot"), st["k_weight"])
    out = dict(q=_normed_rotated(st, st["q"], st.get("q_rot"), st.get("q_weight")).to(torch.bfloat16), rows=phys * page + off)
    if case["keys"]:
        out["keys"] = k.to(torch.bfloat16)
    for x, new in (("k", k), ("v", st["v"].float() if "v" in st else None)):
        if new is None:
            continue
        cache = st[x + "_cache"]
        if case["fp8"]:
            codes, scale = _quantised(new)
            cache.view(torch.uint8)[phys, :, off] = codes.view(torch.uint8)
            st[x + "_scale"][phys, :, off] = scale
            out[x + "_scale"] = st[x + "_scale"]
        else:
            cache[phys, :, off] = new.to(torch.bfloat16)
        out[x + "_cache"] = cache
    return out


def _plain_rows(st, x, b, n):
    """The first n cached rows of sequence b as [kv_heads, n, d] in fp32."""
    pages = st["table"][b, :-(-n // st["case"]["page"])].long()
    if st["case"]["fp8"]:
        rows = st[x + "_cache"].view(torch.uint8)[pages].view(FP8).float() * st[x + "_scale"][pages][..., None]
    else:
        rows = st[x + "_cache"][pages].float()
    return rows.transpose(0, 1).flatten(1, 2)[:, :n]


def _plain_cache_read(st):
    out = {}
    for x in ("k", "v"):
        if x + "_cache" in st:
            rows = [_plain_rows(st, x, b, n).transpose(0, 1) for b, n in enumerate(st["new"])]
            out[x] = torch.cat(rows).to(torch.bfloat16)
    return out


def _plain_sequence(case, q, k, v, scale, causal):
    """q [n, H, d_qk], k and v [kv_heads, c, d] in fp32: the attention of the last n of c tokens, by blocks of rows."""
    n, H = q.shape[:2]
    Hkv, c = k.shape[:2]
    outs, lses = [], []
    rows = max(1, min(n, (1 << 29) // max(1, H * c)))
    for j in range(0, n, rows):
        r = min(rows, n - j)
        last = c - n + j + r if causal else c          # keys any of these rows attends to
        last = max(last, 1)
        qb = q[j:j + r].float().view(r, Hkv, H // Hkv, -1).permute(1, 2, 0, 3).reshape(Hkv, H // Hkv * r, -1)
        s = torch.bmm(qb, k[:, :last].transpose(1, 2)).mul_(scale).view(Hkv, H // Hkv, r, last)
        if causal:
            at, t = torch.arange(last, device=DEV), c - n + j + torch.arange(r, device=DEV)[:, None]
            seen = at <= t
            if case["k_swa"]:
                seen &= (at < case["k_sink"]) | (at > t - case["k_swa"])
            s.masked_fill_(~seen, float("-inf"))
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.bmm(p.view(Hkv, -1, last), v[:, :last]).view(Hkv, H // Hkv, r, -1) / total
        outs.append(o.permute(2, 0, 1, 3).reshape(r, H, -1).to(torch.bfloat16))
        lses.append((total.log() + top)[..., 0].permute(2, 0, 1).reshape(r, H))
    return torch.cat(outs), torch.cat(lses)


def _plain_attn(st):
    case, at = st["case"], st["at"]
    outs, lses = [], []
    for b, n in enumerate(st["new"]):
        q = st["q"][at[b]:at[b + 1]]
        if case["op"] == "prefill":
            lo, hi = st["kv_at"][b], st["kv_at"][b + 1]
            k, v = (st[x][lo:hi].float().transpose(0, 1).contiguous() for x in ("k", "v"))
        else:
            k, v = (_plain_rows(st, x, b, st["ctx_list"][b]).contiguous() for x in ("k", "v"))
        o, l = _plain_sequence(case, q, k, v, _scale(case), case.get("causal", True))
        outs.append(o)
        lses.append(l)
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def _scale(case):
    return (case["d"] if case["op"] == "chunk" else case["d_qk"]) ** -0.5


# ------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"norm_append": _plain_norm_append, "cache_read": _plain_cache_read}.get(op, _plain_attn)(st)
    from paper_2608_01662_amd import lsa
    if op == "norm_append":
        latent, rot = case["kind"] == "latent", case["rot_dim"]
        prm = lsa.AppendParams(n_heads=case["heads"], n_kv_heads=case["kv_heads"], d_k=case["d"], d_v=0 if latent else case["d"],
                               rot_start=case["d"] - rot if latent else 0, rot_dim=rot, interleaved=case["interleaved"],
                               fp8=case["fp8"])
        # a decode step names its tokens by the context lengths, a chunk of prompts by sequence and position
        where = dict(ctx_len=st["ctx"]) if case["decode"] else dict(seq=st["seq"], pos=st["pos"])
        q, keys, rows = lsa.norm_append(prm, st["k"], st["k_cache"], q_weight=st.get("q_weight"), k_weight=st["k_weight"], eps=EPS,
                                        page_table=st["table"], rope=st["rope"], k_rot=st.get("k_rot"), v=st.get("v"),
                                        v_cache=st.get("v_cache"), k_scale=st.get("k_scale"), v_scale=st.get("v_scale"),
                                        q=st["q"], q_rot=st.get("q_rot"), k_out=case["keys"], rows=True, **where)
        out = dict(q=q, rows=rows)
        if case["keys"]:
            out["keys"] = keys
        out.update({x: st[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale") if x in st})
        return out
    if op == "cache_read":
        prm = lsa.CacheReadParams(n_kv_heads=case["kv_heads"], d_k=case["d"], d_v=case["d"] if "v_cache" in st else 0, fp8=case["fp8"])
        k, v = lsa.cache_read(prm, st["k_cache"], st["cu"], st["at"][-1], page_table=st["table"], v_cache=st.get("v_cache"),
                              k_scale=st.get("k_scale"), v_scale=st.get("v_scale"))
        return dict(k=k) if v is None else dict(k=k, v=v)
    if op == "prefill":
        prm = lsa.PrefillAttnParams(n_heads=case["heads"], n_kv_heads=case["kv_heads"], d_qk=case["d_qk"], d_v=case["d_v"],
                                    sm_scale=_scale(case), causal=case["causal"], k_sink=case["k_sink"], k_swa=case["k_swa"])
        out, lse = lsa.prefill_attn(prm, st["q"], st["k"], st["v"], st["cu"], st["cu_kv"])
    else:
        prm = lsa.DecodeAttnParams(n_heads=case["heads"], n_kv_heads=case["kv_heads"], d_qk=case["d"], d_v=case["d"], latent=False,
                                   sm_scale=_scale(case), fp8=case["fp8"], k_sink=case["k_sink"], k_swa=case["k_swa"])
        out, lse = lsa.chunk_attn(prm, st["q"], st["k_cache"], st["v_cache"], st["cu"], st["ctx"], page_table=st["table"],
                                  k_scale=st.get("k_scale"), v_scale=st.get("v_scale"))
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------------------------------ work
def _pairs(case):
    """(query, key) pairs of one head that count."""
    sink, swa, total = case["k_sink"], case["k_swa"], 0
    for before, n in zip(*_lengths(case)):
        if not case.get("causal", True):
            total += n * (before + n)
        elif not swa:
            total += n * before + n * (n + 1) // 2
        else:
            for t in (range(before, before + n)):
                window = min(t + 1, swa)
                total += window + min(sink, t + 1 - window)
    return total


def work(case):
    before, new = _lengths(case)
    n, Hkv = sum(new), case["kv_heads"]
    if case["op"] == "prefill":
        H, d_qk, d_v = case["heads"], case["d_qk"], case["d_v"]
        kv = n + sum(before)
        return dict(bytes=n * H * ((d_qk + d_v) * 2 + 4) + kv * Hkv * (d_qk + d_v) * 2, flops=2.0 * H * (d_qk + d_v) * _pairs(case))
    d, each = case["d"], 1 if case["fp8"] else 2
    kinds = 1 if case.get("kind") == "latent" else 2
    row = kinds * Hkv * (d * each + (4 if case["fp8"] else 0))
    if case["op"] == "cache_read":
        return dict(bytes=n * (row + kinds * Hkv * d * 2), flops=n * kinds * Hkv * d)
    if case["op"] == "norm_append":
        H, rot = case["heads"], case["rot_dim"]
        normed = Hkv * (LATENT if kinds == 1 else d) + (0 if kinds == 1 else H * d)
        # in: queries, keys, values, an angle row and two indexes per token; out: queries, cache rows, scales, keys, rows
        return dict(bytes=n * (2 * H * d * 2 + kinds * Hkv * d * 2 + row + (Hkv * d * 2 if case["keys"] else 0) + 4 * rot + 8 + 8),
                    flops=n * (4 * normed + 3 * rot * (H + Hkv)))
    H, read = case["heads"], 0
    for a, b in zip(before, new):       # (of a window, the rows that some new token attends to)
        read += a + b if not case["k_swa"] else min(a + b, case["k_sink"] + case["k_swa"] + b - 1)
    return dict(bytes=n * H * (2 * d * 2 + 4) + read * row, flops=4.0 * H * d * _pairs(case))


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The outputs in 64 bits from the operators' definitions, sequence by sequence and head by head."""
    st = prepare(case, seed)
    return {"norm_append": _exact_norm_append, "cache_read": _exact_cache_read}.get(case["op"], _exact_attn)(st)


def _exact_norm_append(st):
    case = st["case"]
    rot, d, page = case["rot_dim"], case["d"], case["page"]
    start = d - rot if case["kind"] == "latent" else 0
    pair = torch.arange(rot // 2, device=DEV)
    one, two = (2 * pair, 2 * pair + 1) if case["interleaved"] else (pair, pair + rot // 2)
    pos = st["pos"].long()

    def turned(x, part, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(2, keepdim=True) / x.shape[2] + EPS) * weight.double()
        if part is not None:
            x = torch.cat([x, part.double()], dim=2)
        y = x.clone()
        c, s = st["rope"][pos, :rot // 2].double()[:, None], st["rope"][pos, rot // 2:].double()[:, None]
        y[:, :, start + one] = x[:, :, start + one] * c - x[:, :, start + two] * s
        y[:, :, start + two] = x[:, :, start + two] * c + x[:, :, start + one] * s
        return y

    row = st["table"][st["seq"].long(), pos // page].long() * page + pos % page
    keys = turned(st["k"], st.get("k_rot"), st["k_weight"])
    out = dict(q=turned(st["q"], st.get("q_rot"), st.get("q_weight")), rows=row)
    if case["keys"]:
        out["keys"] = keys
    for x, new in (("k", keys), ("v", st["v"].double() if "v" in st else None)):
        if new is None:
            continue
        shape = st[x + "_cache"].shape                      # [n_phys, kv_heads, page, d]
        rows = torch.zeros((shape[0] * page, shape[1], d), dtype=torch.float64, device=DEV)
        if case["fp8"]:
            top = new.abs().amax(2)
            scale = torch.where(top > 0, top / 448, 1.0)
            scales = torch.zeros((shape[0] * page, shape[1]), dtype=torch.float64, device=DEV)
            scales[row] = scale
            out[x + "_scale"] = scales.view(shape[0], page, shape[1]).transpose(1, 2).contiguous()
            new = new / scale[:, :, None]
        rows[row] = new
        out[x + "_cache"] = rows.view(shape[0], page, shape[1], d).transpose(1, 2).contiguous()
    return out


def _exact_row(st, x, b, head, n):
    """Cached rows of one head, position by position."""
    page = st["case"]["page"]
    s = torch.arange(n, device=DEV)
    phys, off = st["table"][b].long()[s // page], s % page
    if st["case"]["fp8"]:
        codes = st[x + "_cache"].view(torch.uint8)[phys, head, off].view(FP8).double()
        return codes * st[x + "_scale"][phys, head, off].double()[:, None]
    return st[x + "_cache"][phys, head, off].double()


def _exact_cache_read(st):
    out = {}
    for x in ("k", "v"):
        if x + "_cache" in st:
            heads = range(st["case"]["kv_heads"])
            out[x] = torch.cat([torch.stack([_exact_row(st, x, b, h, n) for h in heads], dim=1) for b, n in enumerate(st["new"])])
    return out


def _exact_attn(st):
    case = st["case"]
    H, Hkv, prefill = case["heads"], case["kv_heads"], case["op"] == "prefill"
    group, causal = H // Hkv, case.get("causal", True)
    d_v = case["d_v"] if prefill else case["d"]
    total = st["at"][-1]
    out = torch.zeros((total, H, d_v), dtype=torch.float64, device=DEV)
    lse = torch.full((total, H), float("-inf"), dtype=torch.float64, device=DEV)
    for b, n in enumerate(st["new"]):
        lo, c = st["at"][b], st["before"][b] + n
        for head in range(Hkv):
            if prefill:
                k0 = st["kv_at"][b]
                k, v = st["k"][k0:k0 + c, head].double(), st["v"][k0:k0 + c, head].double()
            else:
                k, v = _exact_row(st, "k", b, head, c), _exact_row(st, "v", b, head, c)
            step = max(1, (1 << 27) // max(c, 1) // group)
            for j in range(0, n, step):
                m = min(step, n - j)
                t = torch.arange(c - n + j, c - n + j + m, device=DEV)[:, None, None]
                end = c - n + j + m if causal else c
                s = torch.arange(end, device=DEV)
                x = torch.matmul(st["q"][lo + j:lo + j + m, head * group:(head + 1) * group].double(), k[:end].T) * _scale(case)
                if causal:
                    hidden = s > t
                    if case["k_swa"]:
                        hidden |= (s >= case["k_sink"]) & (s <= t - case["k_swa"])
                    x.masked_fill_(hidden, float("-inf"))
                l = torch.logsumexp(x, dim=2)
                lse[lo + j:lo + j + m, head * group:(head + 1) * group] = l
                out[lo + j:lo + j + m, head * group:(head + 1) * group] = torch.matmul(torch.exp(x - l[..., None]), v[:end])
    return dict(out=out, lse=lse)
