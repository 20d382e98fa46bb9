"""How far attention over a paged cache may be off, as a norm over a row and head: a limit that one missing key exceeds.

A weight p_j that carries a relative error d_j moves the result by sum_j p_j d_j (v_j - o) (for the part of d_j that is in the sum of the
weights too) or sum_j p_j d_j v_j (for the part that is not: the weights' last rounding).  The d_j are roundings of different
numbers and the v_j random vectors of many elements, nearly orthogonal, so the norm is that of a sum of independent terms,
d * R with R^2 = sum_j p_j^2 (|v_j|^2 + |o|^2), where |d_j| <= d.  Roundings spread evenly have a mean square of d^2 / 3 at most,
which leaves a factor of 1.7 for what is not independent; a quarter more is allowed for rows of few keys.  A key of weight p that is
missing moves the result by p |v_j - o|: with n keys of like weights 1 / sqrt(n) of R, against 2^-8 (bf16 weights) of it.
"""
from __future__ import annotations

import torch

import paged_reference as P


def reference(q, contents, layout, scale, group, exists=None):
    """(out [n_tokens, n_heads, head_dim], R and the largest sum_d |q_d k_jd| |scale| of a key [n_tokens, n_heads]) in 64 bits.  exists:
    for each sequence which of its keys lie on pages that exist.  Rows without a place, or without a key: zeros."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    R, terms = (torch.zeros(q.shape[:2], dtype=torch.float64) for _ in range(2))
    for s, (n, length) in enumerate(zip(layout.new, layout.length)):
        lo = max(0, n - length)                                 # rows without a place
        if n == lo:
            continue
        r = slice(int(layout.first[s]) + lo, int(layout.first[s]) + n)
        k, v = contents[s]
        qs = q[r].double().unflatten(1, (k.shape[0], group))    # [rows, kv heads, group, head_dim]
        seen = torch.arange(length) <= torch.arange(length - (n - lo), length).unsqueeze(1)
        if exists is not None:
            seen = seen & exists[s]
        x = torch.einsum("rkgd,kjd->rkgj", qs, k) * scale
        w = torch.nan_to_num(torch.softmax(x.masked_fill(~seen[:, None, None], float("-inf")), -1), nan=0.0)
        o = torch.einsum("rkgj,kjd->rkgd", w, v)
        size = torch.einsum("rkgj,kj->rkg", w ** 2, (v ** 2).sum(-1)) + (w ** 2).sum(-1) * (o ** 2).sum(-1)
        most = (torch.einsum("rkgd,kjd->rkgj", qs.abs(), k.abs()) * abs(scale)).masked_fill(~seen[:, None, None], 0.0).amax(-1)
        out[r], R[r], terms[r] = o.flatten(1, 2), size.sqrt().flatten(1), most.flatten(1)
    return out, R, terms


def limit(out, R, terms, score_rel, weight_rel, out_dtype):
    """Largest norm of the error of a row and head: weights off by weight_rel, scores by score_rel of `terms`, the result rounded once."""
    return out.norm(dim=-1) * torch.finfo(out_dtype).eps / 2 + 1.25 * R * (weight_rel + torch.expm1(score_rel * terms)) + 1e-30


def rels(hd, q_dtype, out_dtype):
    """(score_rel, weight_rel) of the arithmetic over a cache in bf16 or 8 bits: sums of head_dim products in fp32, scales and base
    change; weights as one bf16 where queries and results are bf16 (which the queries then are already), else both with 16 bits."""
    score, weight = (hd + 2 + 8) * 2.0 ** -24, 2.0 ** -18
    if q_dtype == out_dtype == torch.bfloat16:
        return score, weight + 2.0 ** -8
    return score + 2.0 ** -16, weight + 2.0 ** -16


def over(got, want, R, terms, hd, q_dtype):
    """Error of each row and head over its limit."""
    return (got.double() - want).norm(dim=-1) / limit(want, R, terms, *rels(hd, q_dtype, got.dtype), got.dtype)


def contents_of(layout, kv_heads, hd, seed):
    """Random K and V of each sequence, bf16 values."""
    g = torch.Generator().manual_seed(seed)
    return [tuple(torch.randn(kv_heads, l, hd, generator=g).bfloat16().double() for _ in range(2)) for l in layout.length]


__all__ = ["P", "reference", "limit", "rels", "over", "contents_of"]
