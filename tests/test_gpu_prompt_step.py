"""The prompt-side operators together, as examples/prompt_step.py and a server use them: norm_append, cache_read, prefill_attn, chunk_attn
and decode_attn over the same caches. Tolerances: tests/prompt_check.py, and where two kernels are compared, the sum of both."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

from paper_2608_01662_amd import lsa
from tests.prompt_check import BF16, DEV, compare, i32, sees

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("prompt_step", os.path.join(ROOT, "examples", "prompt_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rows(layer, x, b, n):
    """The first n cached rows [HKV, n, D] of sequence b in float64."""
    page = layer.k.shape[2]
    pages = layer.pages.table[b, :-(-n // page)].long()
    cache = getattr(layer, x)
    scale = layer.scales.get(x + "_scale")
    r = cache[pages].double() if scale is None else cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * scale[pages].double()[..., None]
    return r.transpose(0, 1).flatten(1, 2)[:, :n]


def test_the_example_runs():
    """Whole prompts, chunks and single tokens: the same keys in bf16, so two outputs of one row differ by no more than both kernels' roundings
    (each within 2.02 * 2^-8 of a bound of |o|, which the largest value bounds)."""
    outs = _example().run(batch=5, prompt=500, chunk=130, steps=3, seed=3)
    lens, a, b, c, steps = outs
    assert a.shape[0] == sum(lens) == c.shape[0] and torch.isfinite(c.float()).all()
    most = 6.0          # largest |v| of 5e6 normal values
    assert float((a.float() - b.float()).abs().max()) <= 2 * 2.1 * 2.0 ** -8 * most
    for one, dec in steps:
        assert float((one.float() - dec.float()).abs().max()) <= 2 * 2.1 * 2.0 ** -8 * most


@pytest.mark.parametrize("fp8", [False, True])
def test_chunks_over_what_was_appended(fp8):
    """Three steps of ragged chunks (one sequence idle, one of single tokens) against 64 bits over the rows that the caches hold."""
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(1)
    pages = m.Pages(4, 2000, DEV)
    layer = m.GroupedLayer(pages, 2000, DEV, fp8)
    done = [0, 0, 0, 0]
    for new in ([300, 1, 0, 65], [129, 1, 640, 1], [1, 1, 1, 700]):
        ctx = [d + n for d, n in zip(done, new)]
        qkv, _ = m.projections(sum(new), g)
        out, lse = layer.chunks(qkv, new, ctx)
        q, _ = layer.append(qkv, **m.places(new, ctx, DEV))      # (again: the same rows, the same values)
        at = 0
        for b, (n, c) in enumerate(zip(new, ctx)):
            k, v = _rows(layer, "k", b, c), _rows(layer, "v", b, c)
            for h in range(layer.HKV):
                hs = slice(4 * h, 4 * h + 4)
                compare(out[at:at + n, hs], lse[at:at + n, hs], q[at:at + n, hs].double(), k[h], v[h], sees(n, c, True, 0, 0), layer.cached.sm_scale, (b, n, c),
                        extra=2 if fp8 else 0)
            at += n
        done = ctx


def test_whole_prompts_over_their_own_keys():
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(2)
    pages = m.Pages(3, 700, DEV)
    layer = m.GroupedLayer(pages, 700, DEV)
    lens = [700, 3, 333]
    qkv, _ = m.projections(sum(lens), g)
    out, lse = layer.prompts(qkv, lens)
    q, keys = layer.append(qkv, keys=True, **m.places(lens, lens, DEV))
    back, values = lsa.cache_read(lsa.CacheReadParams(8, 128, 128), layer.k, m.offsets(lens, DEV), sum(lens), page_table=pages.table, v_cache=layer.v)
    assert torch.equal(back, keys) and torch.equal(values, layer.heads(qkv)[2])
    at = 0
    for b, n in enumerate(lens):
        for h in range(8):
            hs = slice(4 * h, 4 * h + 4)
            compare(out[at:at + n, hs], lse[at:at + n, hs], q[at:at + n, hs].double(), back[at:at + n, h].double(), values[at:at + n, h].double(),
                    sees(n, n, True, 0, 0), layer.prefill.sm_scale, (b, n))
        at += n


def test_latent_chunks_unabsorbed():
    """The latent layer's second chunk: rows read back, up-projected, attended to, against 64 bits of the same queries, keys and values; and the rows
    that are read back are those that the cache holds."""
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(4)
    pages = m.Pages(3, 600, DEV)
    layer = m.LatentLayer(pages, 600, DEV)
    done = [0, 0, 0]
    for new in ([200, 1, 64], [300, 2, 1]):
        ctx = [d + n for d, n in zip(done, new)]
        _, x = m.projections(sum(new), g)
        (out, lse), (q, k, v) = layer.chunks(x, new, ctx)
        at = kv_at = 0
        for b, (n, c) in enumerate(zip(new, ctx)):
            for h in range(0, 64, 9):
                compare(out[at:at + n, h:h + 1], lse[at:at + n, h:h + 1], q[at:at + n, h:h + 1].double(), k[kv_at:kv_at + c, h].double(),
                        v[kv_at:kv_at + c, h].double(), sees(n, c, True, 0, 0), layer.prefill.sm_scale, (b, n, c, h))
            held = layer.kv[pages.table[b].long()].flatten(0, 1)[:c, 512:]
            assert torch.equal(k[kv_at:kv_at + c, 5, 128:], held)
            at, kv_at = at + n, kv_at + c
        done = ctx


def test_a_captured_step():
    """norm_append, chunk_attn and cache_read captured once, replayed for later steps with the lengths and positions in the captured buffers:
    every replay gives what the same calls give outside the graph, with other work of the program between."""
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(6)
    pages = m.Pages(3, 2100, DEV)
    layer, other = (m.GroupedLayer(pages, 2100, DEV) for _ in range(2))
    new = [40, 1, 7]
    seq = m.places(new, new, DEV)["seq"]
    cu = m.offsets(new, DEV)
    qkv = m.projections(sum(new), g)[0]
    pos, ctx = torch.zeros(sum(new), dtype=torch.int32, device=DEV), i32(new)
    prm = layer.cached
    size = lsa.chunk_attn_workspace_size(prm, 3, sum(new), pages.table.shape[1], 64)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    read = lsa.CacheReadParams(8, 128, 128)

    def step(layer, **kw):
        q, _ = layer.append(qkv, seq=seq, pos=pos)
        out, lse = lsa.chunk_attn(prm, q, layer.k, layer.v, cu, ctx, page_table=pages.table, **kw)
        last = ctx - 1
        k, v = lsa.cache_read(read, layer.k, torch.arange(4, dtype=torch.int32, device=DEV), 3, page_table=pages.table, start=last, v_cache=layer.v)
        return out, lse, k, v

    def set_to(lens):
        pos.copy_(m.places(new, lens, DEV)["pos"])
        ctx.copy_(i32(lens))
    set_to([40, 1, 7])
    step(layer, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(layer, workspace=ws)
    for lens in ([40, 1, 7], [80, 2, 14], [2000, 900, 21], [2040, 901, 28]):
        set_to(lens)
        qkv.copy_(m.projections(sum(new), g)[0])
        graph.replay()
        want = step(other)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), lens


def test_steps_on_two_streams():
    """Two layers' steps at once on two streams, each with caches and workspaces of its own, give what they give one after the other."""
    m = _example()
    g = torch.Generator(device=DEV).manual_seed(7)
    pages = m.Pages(2, 3000, DEV)
    work = []
    for _ in range(2):
        layer = m.GroupedLayer(pages, 3000, DEV)
        first, later = m.projections(2990 + 2000, g)[0], m.projections(31, g)[0]
        layer.chunks(first, [2990, 2000], [2990, 2000])
        work.append((layer, later, [t.clone() for t in layer.chunks(later, [1, 30], [2991, 2030])], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        outs = []
        for layer, later, want, s in work:
            with torch.cuda.stream(s):
                outs.append(layer.chunks(later, [1, 30], [2991, 2030]))
        torch.cuda.synchronize()
        for (_, _, want, _), got in zip(work, outs):
            assert all(torch.equal(x, y) for x, y in zip(want, got))
