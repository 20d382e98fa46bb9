"""Plain 64-bit CPU forms of the 4-bit paged cache: value = code (e2m1) * block scale (e4m3, 16 elements) * scale (fp32, a row)."""
from __future__ import annotations

import torch

import paged_reference as P

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
E4M3 = torch.arange(0, 0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn).double()      # the values that are not negative, in order: 0 .. 448


def nearest(y, values):
    """Index of the nearest of the increasing values to each y >= 0; halfway between two the even index; beyond the last the last."""
    at = torch.searchsorted(values, y.contiguous()).clamp(1, len(values) - 1)
    below, above = y - values[at - 1], values[at] - y
    return torch.where((below > above) | ((below == above) & (at % 2 == 0)), at, at - 1)


def quantise(x):
    """(codes 0..15 [.., d], block codes [.., d / 16], scales fp32 [..]) of rows along the last axis, decided in 64 bits."""
    x = x.double()
    finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
    scale = (finite.amax(-1).float() / torch.tensor(2688.0)).float()
    s = torch.where(scale > 0, scale, 1.0).double().unsqueeze(-1)
    part = x.unflatten(-1, (-1, 16))
    top = torch.where(torch.isinf(part).any(-1), finite.amax(-1, keepdim=True), finite.unflatten(-1, (-1, 16)).amax(-1))
    block = nearest(top / (6 * s), E4M3)
    unit = E4M3[block].unsqueeze(-1) * s.unsqueeze(-1)
    y = torch.nan_to_num(part, nan=0.0).abs() / torch.where(unit > 0, unit, 1.0)
    code = nearest(y, E2M1) | torch.where(part < 0, 8, 0)
    dead = (scale == 0).unsqueeze(-1)
    block = torch.where(dead, 0, block)
    code = torch.where(dead.unsqueeze(-1) | (block == 0).unsqueeze(-1), 0, code)
    return code.flatten(-2).to(torch.uint8), block.to(torch.uint8), scale


def values(code, block, scale):
    """What the parts stand for, in 64 bits."""
    v = E2M1[(code & 7).long()] * (1 - 2 * (code >> 3).double())
    return v * E4M3[block.long()].repeat_interleave(16, -1) * scale.double().unsqueeze(-1)


def stored(x):
    """What a cache in 4 bits gives back for rows x, in fp32: code times block scale is exact, one rounding."""
    return values(*quantise(x)).float()


def pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def unpack(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def fill(cache, layout, layer=0, seed=1, k_gain=1.0, v_gain=1.0):
    """Random contents of every used place, written into the pools (not through append); everything else: NaN scales and block scales,
    codes of ones.  Returns K and V [n_kv_heads, length, head_dim] of each sequence in 64 bits."""
    c = cache.cfg
    pool = cache.layer(layer)
    g = torch.Generator().manual_seed(seed)
    host = {n: torch.full(t.shape, float("nan")) if t.dtype == torch.float32 else torch.full(t.shape, 0x7f if n.endswith("block") else 0xff, dtype=torch.uint8)
            for n, t in pool.items()}
    out = []
    for s, l in enumerate(layout.length):
        kv = {}
        for n, gain in (("k", k_gain), ("v", v_gain)):
            code, block, scale = quantise(torch.randn(c.n_kv_heads, l, c.head_dim, generator=g) * gain)
            kv[n] = values(code, block, scale)
            for p0 in range(0, l, c.page_len):
                page, p1 = int(layout.pages[s, p0 // c.page_len]), min(p0 + c.page_len, l)
                host[n][page, :, :p1 - p0] = pack(code)[:, p0:p1]
                host[n + "_block"][page, :, :p1 - p0] = block[:, p0:p1]
                host[n + "_scale"][page, :, :p1 - p0] = scale[:, p0:p1]
        out.append((kv["k"], kv["v"]))
    for n, t in pool.items():
        (t if t.dtype in (torch.float32, torch.uint8) else t.view(torch.uint8)).copy_(host[n])
    return out


def fill_any(cache, layout, **kw):
    return fill(cache, layout, **kw) if cache.cfg.dtype == 6 else P.fill(cache, layout, **kw)
