"""The serving steps of examples/serve_step.py: while a context fits the index budget, the sparse attention lists every
position and agrees with the attention over the whole latent cache; the dense layer agrees with plain attention over
what its fp8 cache holds."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

from tests import parity as P

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_sparse_and_dense_agree_within_the_index_budget():
    """Two kernels of bf16 outputs and weights, each within parity's rule of the exact result: within twice that."""
    m = _example()
    outs = m.run(batch=5, prompt=900, steps=4, seed=3)
    for ctx, dense, sparse, whole in outs:
        assert int(ctx.max()) <= 4 + 256 + 768
        a, b = sparse.float().cpu(), whole.float().cpu()
        assert torch.isfinite(dense.float()).all() and torch.isfinite(a).all()
        assert float((a - b).abs().max()) <= 2 * P.ATOL_O
        assert float((a - b).norm() / b.norm()) <= 2 * P.RTOL_O


def test_dense_layer_against_plain_attention():
    """One more step of the dense layer against softmax attention in 64 bits over the dequantised cache and the rotated
    queries: parity's rule."""
    m = _example()
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)
    pages = m.Pages(3, 300, dev)
    layer = m.DenseLayer(pages, 300, dev)
    for n in range(1, 4):       # three tokens of each sequence, one after the other
        qkv, _ = m.projections(3, g)
        ctx = torch.full((3,), n, dtype=torch.int32, device=dev)
        out = layer.step(qkv, ctx)
    q = layer.append(qkv, ctx_len=ctx).double().cpu()      # (again: the same rows, the same values)
    for b in range(3):
        page = int(pages.table[b, 0])
        k = (layer.k[page, :, :3].float() * layer.ks[page, :, :3, None]).double().cpu()
        v = (layer.v[page, :, :3].float() * layer.vs[page, :, :3, None]).double().cpu()
        for h in range(32):
            p = torch.softmax(k[h // 4] @ q[b, h] * layer.at.sm_scale, 0)
            ref = p @ v[h // 4]
            got = out[b, h].double().cpu()
            assert float((got - ref).abs().max()) <= P.ATOL_O and float((got - ref).norm() / ref.norm()) <= P.RTOL_O
