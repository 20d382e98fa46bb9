"""Plain 64-bit CPU forms of the paged-cache operators and of token selection, and the error bounds their tests use."""
from __future__ import annotations

import math

import torch

TOP = {"int8": 127.0, "e4m3": 448.0}
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}


class Layout:
    """Sequences of a call: new tokens and length of each, pages handed out in a shuffled order, some left over."""

    def __init__(self, new, length, page_len, seed=0, spare_pages=3, spare_columns=1, start=0, tail=0):
        assert len(new) == len(length)
        g = torch.Generator().manual_seed(seed)
        self.new, self.length, self.page_len = list(new), list(length), page_len
        need = [(l + page_len - 1) // page_len for l in length]
        self.n_pages = sum(need) + spare_pages
        self.columns = max(need + [1]) + spare_columns
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.pages = torch.full((len(new), self.columns), -1, dtype=torch.int32)       # unused entries are no pages
        for s, n in enumerate(need):
            for i in range(n):
                self.pages[s, i] = order.pop()
        first = [start]
        for n in new:
            first.append(first[-1] + n)
        self.first = torch.tensor(first, dtype=torch.int32)
        self.n_tokens = first[-1] + tail                     # `start` rows of padding ahead, `tail` rows behind
        self.len = torch.tensor(self.length, dtype=torch.int32)

    def places(self):
        """(row, sequence, position) of every row that has a place."""
        for s, n in enumerate(self.new):
            for i in range(n):
                p = self.length[s] - n + i
                if p >= 0:
                    yield int(self.first[s]) + i, s, p

    def slot(self, s, p):
        return int(self.pages[s, p // self.page_len]), p % self.page_len

    def batch(self, device="cuda", max_len=None):
        from paper_2307_02628_b200 import binding
        return binding.CacheBatch(self.pages.to(device), self.first.to(device), self.len.to(device), self.n_tokens,
                                  max(max(self.new), 1), max(self.length) if max_len is None else max_len)


def make_cache(layout, n_heads, n_kv_heads, head_dim, dtype, n_layers=1, **kw):
    from paper_2307_02628_b200 import binding
    return binding.PagedCache(n_layers, n_heads, n_kv_heads, head_dim, layout.page_len, layout.n_pages, max_seqs=max(8, len(layout.new)),
                              max_tokens=max(8, layout.n_tokens), dtype=dtype, **kw)


def round_e4m3(y):
    """Nearest value with 3 fraction bits and exponents from -6, ties to even, at most 448 in magnitude."""
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def quantise(x, dtype):
    """(values of the codes, scales in fp32) of fp32 rows along the last axis, decided in 64 bits."""
    x = x.double()
    finite = torch.isfinite(x)
    scale = (torch.where(finite, x.abs(), 0.0).amax(-1) / TOP[dtype]).float()
    y = x / torch.where(scale > 0, scale, 1.0).double().unsqueeze(-1)
    y = torch.nan_to_num(y, nan=0.0).clamp(-TOP[dtype], TOP[dtype])
    y = torch.round(y) if dtype == "int8" else round_e4m3(y)
    return torch.where((scale > 0).unsqueeze(-1), y, 0.0), scale


def stored(x, dtype):
    """What a cache of `dtype` gives back for rows x, in fp32."""
    if dtype in TOP:
        codes, scale = quantise(x, dtype)
        return codes.float() * scale.unsqueeze(-1)
    most = torch.finfo(TORCH[dtype]).max
    return torch.nan_to_num(x.float(), nan=0.0, posinf=most, neginf=-most).clamp(-most, most).to(TORCH[dtype]).float()


def fill(cache, layout, layer=0, seed=1, k_gain=1.0, v_gain=1.0):
    """Random contents of every used place, written into the pools (not through append), everything else NaN bytes; returns
    what the cache then holds, as 64-bit K and V [n_kv_heads, length, head_dim] per sequence."""
    c = cache.cfg
    dtype = {0: "fp32", 1: "bf16", 3: "int8", 4: "e4m3"}[c.dtype]
    pool = cache.layer(layer)
    g = torch.Generator().manual_seed(seed)
    out = []
    host = {}
    for n in pool:
        host[n] = torch.full(pool[n].shape, float("nan"), dtype=torch.float32)
        if n in ("k", "v") and dtype == "int8":
            host[n].fill_(-128)
    for s, l in enumerate(layout.length):
        kv = {}
        for n, gain in (("k", k_gain), ("v", v_gain)):
            x = torch.randn(c.n_kv_heads, l, c.head_dim, generator=g) * gain
            if dtype in TOP:
                codes, scale = quantise(x, dtype)
                kv[n] = codes.double() * scale.double().unsqueeze(-1)
            else:
                codes = x.to(TORCH[dtype]).float()
                kv[n] = codes.double()
            for p0 in range(0, l, c.page_len):
                page, p1 = int(layout.pages[s, p0 // c.page_len]), min(p0 + c.page_len, l)
                host[n][page, :, :p1 - p0] = codes[:, p0:p1].float()
                if dtype in TOP:
                    host[n + "_scale"][page, :, :p1 - p0] = scale[:, p0:p1]
        out.append((kv["k"], kv["v"]))
    for n in pool:
        pool[n].copy_(host[n].to(pool[n].dtype).to(pool[n].device) if pool[n].dtype != torch.float8_e4m3fn else
                      host[n].to(torch.float8_e4m3fn).to(pool[n].device))
    return out


def attention(q, contents, layout, scale, group):
    """out [n_tokens, n_heads, head_dim] in 64 bits (rows without a place: zeros), and what `bound` needs."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    spread = torch.zeros(q.shape, dtype=torch.float64)        # sum_j p_j |v_j|
    terms = torch.zeros(q.shape[:2], dtype=torch.float64)     # largest scale * sum_d |q_d k_jd| of a row
    reach = torch.zeros(q.shape[:2], dtype=torch.float64)     # number of keys times their largest |v|
    for r, s, p in layout.places():
        k, v = contents[s]
        k, v = k[:, :p + 1], v[:, :p + 1]
        qr = q[r].double().view(k.shape[0], group, -1)
        w = torch.softmax(torch.einsum("kgd,kjd->kgj", qr, k) * scale, -1)
        out[r] = torch.einsum("kgj,kjd->kgd", w, v).reshape(out[r].shape)
        spread[r] = torch.einsum("kgj,kjd->kgd", w, v.abs()).reshape(out[r].shape)
        terms[r] = (torch.einsum("kgd,kjd->kgj", qr.abs(), k.abs()) * abs(scale)).amax(-1).reshape(-1)
        reach[r] = (v.abs().amax((1, 2)) * (p + 1)).repeat_interleave(group)
    return out, (spread, terms, reach)


def bound(out, parts, score_rel, weight_rel, out_dtype):
    """Largest error of an output.  A score is off by at most score_rel * terms, so every weight p_j by a factor within
    exp(+-2 score_rel terms) (numerator and sum), times 1 +- weight_rel: |error| <= spread * (e^(2 score_rel terms) - 1 + weight_rel) to first
    order (doubled for the rest), and the rounding to the output's type is half a step.

    Where weights enter as sums of two fp16 numbers (8-bit caches), weights below 2^-14 lie on fp16's fixed grid of 2^-24, so each is also
    off by up to 2^-25 of the unit, in which the largest weight times scale is at least 2^7: with a largest code c that key's
    weight moves by at most 2^-32 and its contribution by 2^-32 times the largest |v| (w_j scale_j c <= the largest |v| after
    the division by the sum), for each of the keys: reach * 2^-32 in all."""
    spread, terms, reach = parts
    rel = torch.expm1(2 * score_rel * terms).unsqueeze(-1) + weight_rel
    return 2 * spread * rel + (out.abs() + spread * rel) * torch.finfo(out_dtype).eps / 2 + reach.unsqueeze(-1) * 2.0 ** -32 + 1e-30


def select(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row's token by the definition, in 64 bits."""
    x = torch.where(torch.isnan(logits), float("-inf"), logits.double())
    m = float(x.max())
    if temperature == 0 or not math.isfinite(m):
        return int((x == m).nonzero()[0])
    x, order = torch.sort(x, descending=True, stable=True)
    w = torch.exp((x - m) / float(temperature))
    n = len(w)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        cum = torch.cumsum(w[:n], 0)
        n = max(1, int((torch.cat([torch.zeros(1, dtype=torch.float64), cum[:-1]]) < top_p * cum[-1]).sum()))
    if min_p > 0:
        n = max(1, min(n, int((w >= min_p).sum())))
    cum = torch.cumsum(w[:n], 0)
    return int(order[min(n - 1, int((cum <= min(max(u, 0.0), 1.0) * cum[-1]).sum()))])
