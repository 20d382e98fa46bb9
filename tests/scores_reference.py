"""Attention over a paged cache with capped, biased and masked scores in plain 64-bit form, and how far the kernels may be off.

The limits are those of paged_bounds, over the keys that a row sees.  Beside them a score may be off by 2^-21 of the cap, or of the largest score of the
call where that is less (a polynomial to 3e-7 of the score up to the cap; beyond it two approximations of 2^-22 in a term of at most 0.42 of the cap),
and by 2^-22 of its bias, a product and a sum in fp32: a sum over keys weighted by their bias.
"""
from __future__ import annotations

import torch

import paged_bounds as B


def visible(layout, s, window=0, lo=None, hi=None):
    """[rows with a place, length]: the keys that the rows of sequence s see."""
    n, length = layout.new[s], layout.length[s]
    p = torch.arange(length - n, length)
    key = torch.arange(length)
    first = torch.zeros(n, dtype=torch.long) if window == 0 else p - window + 1
    last = p.clone()
    r = slice(int(layout.first[s]), int(layout.first[s]) + n)
    if lo is not None:
        first = torch.maximum(first, lo[r].long())
    if hi is not None:
        last = hi[r].long()
    see = (key >= first.unsqueeze(1)) & (key <= last.unsqueeze(1))
    return see[max(0, n - length):]


def reference(q, contents, layout, scale, group, exists=None, cap=0.0, slopes=None, window=0, lo=None, hi=None):
    """(out, R, terms, Rb, most): as paged_bounds.reference, R with every key's weight times its bias, the largest visible score before the cap."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    R, terms, Rb = (torch.zeros(q.shape[:2], dtype=torch.float64) for _ in range(3))
    largest = 0.0
    for s, (n, length) in enumerate(zip(layout.new, layout.length)):
        skip = max(0, n - length)                               # rows without a place
        if n == skip:
            continue
        r = slice(int(layout.first[s]) + skip, int(layout.first[s]) + n)
        k, v = contents[s]
        qs = q[r].double().unflatten(1, (k.shape[0], group))    # [rows, kv heads, group, head_dim]
        seen = visible(layout, s, window, lo, hi)
        if exists is not None:
            seen = seen & exists[s]
        x = torch.einsum("rkgd,kjd->rkgj", qs, k) * scale
        largest = max(largest, float(x.abs().max()))
        if cap:
            x = cap * torch.tanh(x / cap)
        far = torch.zeros_like(x)
        if slopes is not None:
            away = (torch.arange(length) - torch.arange(length - (n - skip), length).unsqueeze(1)).abs().double()
            away = away - torch.where(seen, away, 1e18).amin(1, keepdim=True)      # what counts is the difference to the nearest visible key
            far = slopes.double().view(1, k.shape[0], group, 1) * away.view(n - skip, 1, 1, length)
            x = x - far
        w = torch.nan_to_num(torch.softmax(x.masked_fill(~seen[:, None, None], float("-inf")), -1), nan=0.0)
        o = torch.einsum("rkgj,kjd->rkgd", w, v)
        size = lambda w: torch.einsum("rkgj,kj->rkg", w ** 2, (v ** 2).sum(-1)) + (w ** 2).sum(-1) * (o ** 2).sum(-1)  # noqa: E731
        most = (torch.einsum("rkgd,kjd->rkgj", qs.abs(), k.abs()) * abs(scale)).masked_fill(~seen[:, None, None], 0.0).amax(-1)
        out[r], R[r], terms[r] = o.flatten(1, 2), size(w).sqrt().flatten(1), most.flatten(1)
        Rb[r] = size(w * far.abs()).sqrt().flatten(1)
    return out, R, terms, Rb, largest


def over(got, want, R, terms, Rb, largest, hd, q_dtype, cap=0.0):
    """Error of each row and head over its limit."""
    lim = B.limit(want, R, terms, *B.rels(hd, q_dtype, got.dtype), got.dtype) + 1.25 * (R * min(cap, largest) * 2.0 ** -21 + Rb * 2.0 ** -22)
    return (got.double() - want).norm(dim=-1) / lim
