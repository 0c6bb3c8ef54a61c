"""float64 reference of the serving operators (cache append with rotation, attention of new tokens over a
whole paged cache), from their formulas; test infrastructure only."""
from __future__ import annotations

import torch


def cache_row(seq, pos, table, page, n_seq, n_phys):
    """Physical cache row of position `pos` of sequence `seq`, -1 if it has none. table: [n_seq][max_pages]
    lists, or None: sequence b has page b alone."""
    if not 0 <= seq < n_seq or pos < 0:
        return -1
    if table is None:
        return seq * page + pos if pos < page and seq < n_phys else -1
    if pos // page >= len(table[seq]):
        return -1
    ph = table[seq][pos // page]
    return ph * page + pos % page if 0 <= ph < n_phys else -1


def rotate(x, start, dim, interleaved, angles_row):
    """x [heads, d] float64 with dims [start, start + dim) rotated; angles_row [dim]: cosines, then sines."""
    y = x.clone()
    for i in range(dim // 2):
        a, b = (start + 2 * i, start + 2 * i + 1) if interleaved else (start + i, start + i + dim // 2)
        c, s = float(angles_row[i]), float(angles_row[dim // 2 + i])
        y[:, a] = x[:, a] * c - x[:, b] * s
        y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def decode_attention(q, rows_k, rows_v, seen, sm_scale):
    """One row: q [heads, d] float64, rows_k / rows_v [n, d] of its key/value head, seen [n] bool.
    Returns (o [heads, d_v], lse [heads], spread [heads, d_v] = sum p |v|, reach = max sum_i |q_i k_i| over the
    scores): the last two bound the rounding errors of a computation in lower precision."""
    k, v = rows_k[seen], rows_v[seen]
    heads = q.shape[0]
    if k.shape[0] == 0:
        z = torch.zeros((heads, rows_v.shape[1]), dtype=torch.float64)
        return z, torch.full((heads,), float("-inf"), dtype=torch.float64), z, 0.0
    s = sm_scale * (q @ k.T)
    top = s.amax(1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(1, keepdim=True)
    reach = sm_scale * float((q.abs() @ k.abs().T).max())
    return (p @ v) / total, (total.log() + top)[:, 0], (p @ v.abs()) / total, reach
