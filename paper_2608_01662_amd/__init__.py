"""LongCat Sparse Attention (LSA) hot path for AMD Instinct MI355X (gfx950).

HIP kernels behind a C-ABI (include/lsa.h, built into liblsa.so) and a thin ctypes binding:
indexer (mean keys, coarse page scores, page top-M, fine token scores, token top-K with sink and
window merge, runs), sparse attention over the resulting index list, reused across layers, appending
rotated keys and values to the paged caches, and attention of new tokens over a whole cache.
"""
from .lsa import (AppendParams, AttnParams, DecodeAttnParams, IndexParams, LSAError, MLA, MQA,  # noqa: F401
                  attn_workspace_size, block_means, cache_append, decode_attn, decode_attn_workspace_size,
                  index_decode, index_prefill, index_workspace_size, lib, sparse_attn, version)
