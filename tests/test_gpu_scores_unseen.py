"""Positions that no row of a sequence sees: their pages need not exist, and what lies there, on a page that others see a part of, may be anything."""
import pytest
import torch

import four_reference as F
import paged_reference as P
import scores_reference as S
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu

CACHES = ("fp32", "bf16", "int8", "e4m3", "e2m1")


def run(cache_dtype, heads, kv_heads, hd, page, new, length, masks, seed=0, io="bf16", **kw):
    """masks(new tokens, length): a sequence's lo and hi, or None.  Whatever lies outside the sequence's first and last visible position is NaN bytes,
    and table entries of pages that lie there as a whole name none."""
    lay = P.Layout(new, length, page, seed=seed)
    cache = P.make_cache(lay, heads, kv_heads, hd, cache_dtype)
    contents = F.fill_any(cache, lay, seed=seed + 1)
    parts = [masks(n, l) for n, l in zip(new, length)]
    lo, hi = (None if parts[0][i] is None else torch.cat([p[i] for p in parts]).to(torch.int32) for i in (0, 1))
    pool = cache.layer(0)
    pages = lay.pages.clone()
    hidden = 0
    for s, (n, l) in enumerate(zip(new, length)):
        seen = S.visible(lay, s, kw.get("window", 0), lo, hi).any(0).nonzero().flatten().tolist()
        first, last = (seen[0], seen[-1]) if seen else (l, -1)
        for column in range((l + page - 1) // page):
            at = torch.arange(column * page, min(l, (column + 1) * page))
            out = (at < first) | (at > last)
            for name, t in pool.items():
                raw = t.view(torch.uint8).view(*t.shape[:3], -1) if t.dim() == 4 else t.view(torch.uint8).view(*t.shape, 4)
                raw[int(pages[s, column]), :, (at % page)[out].cuda()] = 0xff
            if bool(out.all()):
                pages[s, column] = (-1, lay.n_pages, -(2 ** 31))[hidden % 3]
                hidden += 1
    q = torch.randn(lay.n_tokens, heads, hd, generator=torch.Generator().manual_seed(seed + 2)).to(P.TORCH[io])
    b = binding.CacheBatch(pages.cuda(), lay.first.cuda(), lay.len.cuda(), lay.n_tokens, max(new), max(length))
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    got = cache.attention(0, q.cuda(), b, scores=binding.Scores(kw.get("cap", 0.0), cuda(kw.get("slopes")), kw.get("window", 0), cuda(lo), cuda(hi))).cpu()
    status = cache.status()
    cache.close()
    assert hidden > 0
    assert status == 0
    want = S.reference(q, contents, lay, hd ** -0.5, heads // kv_heads, None, lo=lo, hi=hi, **kw)
    over = S.over(got, *want, hd, q.dtype, kw.get("cap", 0.0))
    assert not bool(torch.isnan(over).any())
    assert float(over.max()) <= 1, float(over.max())


def nothing(n, l):
    return None, None


def late(n, l):
    """Everything from somewhere in the middle on."""
    return torch.full((n,), l // 2 + 3).clamp(max=l - n), None


def early(n, l):
    """The first positions only, the rows' own not among them."""
    return None, torch.full((n,), l // 3 + 1)


def between(n, l):
    return torch.full((n,), l // 3 + 5), torch.full((n,), l // 2 + 2) + torch.arange(n) % 3


FEW = ([1, 2, 1], [700, 331, 90])
MANY = ([70, 300], [700, 900])


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("page", [8, 16, 64])
@pytest.mark.parametrize("hd,heads,kv_heads", [(64, 4, 4), (128, 6, 2), (32, 2, 1)])
@pytest.mark.parametrize("new,length", [FEW, MANY], ids=["few", "many"])
def test_unseen_positions(cache_dtype, page, hd, heads, kv_heads, new, length):
    slopes = 2.0 ** (-8.0 * torch.arange(1, heads + 1) / heads)
    for i, (masks, kw) in enumerate(((nothing, dict(window=1)), (nothing, dict(window=37, cap=5.0)), (nothing, dict(window=64)), (late, dict(slopes=slopes)), (early, dict()),
                                     (between, dict(cap=3.0, slopes=slopes)))):
        run(cache_dtype, heads, kv_heads, hd, page, new, length, masks, seed=i, **kw)


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e2m1"])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
def test_unseen_positions_of_split_keys(cache_dtype, io):
    for new, length in (([65], [5001]), ([1, 3], [9001, 4100])):
        for masks, kw in ((nothing, dict(window=2500)), (late, dict()), (early, dict()), (between, dict())):
            run(cache_dtype, 4, 1, 128, 16, new, length, masks, seed=len(new), io=io, **kw)
