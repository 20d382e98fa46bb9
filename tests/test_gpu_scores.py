"""Attention over a paged cache with capped, biased and masked scores against the 64-bit form, row by row (see scores_reference)."""
import pytest
import torch

import four_reference as F
import paged_reference as P
import scores_reference as S
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu

CACHES = ("fp32", "bf16", "int8", "e4m3", "e2m1")


def run(cache_dtype, heads, kv_heads, hd, page, new, length, scale=None, seed=0, io="bf16", out_dtype=None, gone=(), max_len=None, max_new=None, k_gain=1.0, q_gain=1.0,
        cap=0.0, slopes=None, window=0, lo=None, hi=None, plain=False, **kw):
    """plain: without changed scores.  lo, hi: functions of the layout.  gone: (sequence, column) of table entries that are made to name no page."""
    lay = P.Layout(new, length, page, seed=seed, **kw)
    cache = P.make_cache(lay, heads, kv_heads, hd, cache_dtype)
    contents = F.fill_any(cache, lay, seed=seed + 1, k_gain=k_gain)
    q = (q_gain * torch.randn(lay.n_tokens, heads, hd, generator=torch.Generator().manual_seed(seed + 2))).to(P.TORCH[io])
    lo, hi = (None if f is None else f(lay).to(torch.int32) for f in (lo, hi))
    pages, exists = lay.pages.clone(), [torch.ones(l, dtype=torch.bool) for l in length]
    for i, (s, column) in enumerate(gone):
        pages[s, column] = (-1, lay.n_pages, 1 << 30)[i % 3]
        exists[s][column * page:(column + 1) * page] = False
    b = binding.CacheBatch(pages.cuda(), lay.first.cuda(), lay.len.cuda(), lay.n_tokens, max_new or max(max(new), 1), max(length) if max_len is None else max_len)
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    sc = None if plain else binding.Scores(cap, cuda(slopes), window, cuda(lo), cuda(hi))
    outs = []
    for _ in range(2):
        outs.append(torch.full(q.shape, 9.0, dtype=P.TORCH[out_dtype or io], device="cuda"))
        cache.attention(0, q.cuda(), b, scale=scale, out=outs[-1], scores=sc)
    status = cache.status()
    cache.close()
    assert torch.equal(*outs)
    assert status == 0 or (gone and status == binding.STATUS_BAD_BATCH)
    want = S.reference(q, contents, lay, hd ** -0.5 if scale is None else scale, heads // kv_heads, exists, cap, slopes, window, lo, hi)
    own = torch.zeros(lay.n_tokens, dtype=torch.bool)
    for s in range(len(new)):
        own[int(lay.first[s]):int(lay.first[s + 1])] = True
    got = outs[0].cpu()
    assert bool((got[~own] == 9).all())                         # padding rows are left as they were
    over = S.over(got, *want, hd, q.dtype, cap)[own]
    assert not bool(torch.isnan(over).any())
    assert float(over.max()) <= 1, (float(over.max()), float(over.median()), int(over.argmax()))


def alibi(heads):
    return 2.0 ** (-8.0 * torch.arange(1, heads + 1) / heads)


def positions(lay):
    """Position of every row (0 where it is padding)."""
    p = torch.zeros(lay.n_tokens, dtype=torch.long)
    for s, (n, l) in enumerate(zip(lay.new, lay.length)):
        p[int(lay.first[s]):int(lay.first[s]) + n] = torch.arange(l - n, l)
    return p


def anything(seed, most):
    """Any number for every row: before the sequence, inside, behind."""
    return lambda lay: torch.randint(-4, most + 5, (lay.n_tokens,), generator=torch.Generator().manual_seed(seed))


def documents(mean, seed, empty=13):
    """First positions of documents packed into each sequence; every so many rows one that sees nothing."""
    def lo(lay):
        g = torch.Generator().manual_seed(seed)
        out = torch.zeros(lay.n_tokens, dtype=torch.long)
        for s, (n, l) in enumerate(zip(lay.new, lay.length)):
            starts = torch.cumsum(torch.randint(1, 2 * mean, (l + 1,), generator=g), 0)
            p = torch.arange(l - n, l)
            i = torch.searchsorted(starts, p, right=True)
            out[int(lay.first[s]):int(lay.first[s]) + n] = torch.where(i > 0, starts[(i - 1).clamp_min(0)], 0)
        out[::empty] = 1 << 20
        return out
    return lo


def prefix(most):
    """Rows see the sequence's first positions even where they lie ahead of them."""
    return lambda lay: torch.maximum(positions(lay), torch.tensor(most - 1))


FEW = ([1, 1, 0, 2, 1, 1, 3], [1, 17, 4, 64, 130, 333, 2])
MANY = ([70, 1, 33, 130, 5], [70, 90, 200, 130, 3])


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("new,length", [FEW, MANY], ids=["few", "many"])
@pytest.mark.parametrize("heads,kv_heads,hd,page", [(4, 4, 64, 16), (6, 2, 128, 32), (3, 1, 32, 8)])
def test_each_change(cache_dtype, new, length, heads, kv_heads, hd, page):
    for i, kw in enumerate((dict(cap=3.0), dict(cap=40.0, q_gain=6.0), dict(slopes=alibi(heads)), dict(window=1), dict(window=50), dict(lo=documents(20, 3)),
                            dict(hi=prefix(40)), dict(hi=prefix(40), slopes=alibi(heads)), dict(lo=anything(5, 60)), dict(hi=anything(6, 100)),
                            dict(lo=anything(5, 60), hi=anything(6, 100), cap=5.0, slopes=alibi(heads), window=90))):
        run(cache_dtype, heads, kv_heads, hd, page, new, length, seed=i, start=1, tail=2, **kw)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io,out_dtype", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "bf16")])
@pytest.mark.parametrize("hd", [64, 128])
def test_types(cache_dtype, io, out_dtype, hd):
    for new, length in (FEW, MANY):
        run(cache_dtype, 2, 1, hd, 16, new, length, io=io, out_dtype=out_dtype, seed=hd, cap=8.0, q_gain=3.0, slopes=alibi(2), lo=anything(5, 60), hi=anything(6, 100))
        run(cache_dtype, 2, 1, hd, 16, new, length, io=io, out_dtype=out_dtype, seed=hd, cap=8.0, q_gain=3.0, slopes=alibi(2), window=33)


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e2m1"])
@pytest.mark.parametrize("hd,heads,page", [(64, 4, 16), (128, 7, 64), (128, 4, 8)])
def test_split_keys(cache_dtype, hd, heads, page):
    # one key head: few blocks, so that the keys are split; ranges that begin late, end early and are empty for whole tiles
    for kw in (dict(cap=20.0, q_gain=3.0), dict(window=1500), dict(lo=documents(400, 2)), dict(slopes=alibi(heads) / 16),
               dict(lo=anything(5, 3000), hi=anything(6, 3300)), dict(hi=prefix(2500), slopes=-alibi(heads) / 200)):
        run(cache_dtype, heads, 1, hd, page, [100, 40, 300, 9, 1], [2900, 2049, 300, 4, 3300], seed=hd, start=2, tail=1, **kw)
        run(cache_dtype, heads, 1, hd, page, [65], [3333], seed=hd + 1, **kw)
        run(cache_dtype, heads, 1, hd, page, [1, 2], [9001, 2560], seed=hd + 3, **kw)
        run(cache_dtype, heads, 1, hd, page, [33, 8], [4097, 2560], seed=hd + 2, max_len=1500, **kw)      # longer than the hint


@pytest.mark.parametrize("cache_dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [1, 63, 64, 65, 127, 128, 129, 256, 300, 2 ** 31 - 1])
def test_borders_of_windows(cache_dtype, window):
    run(cache_dtype, 2, 2, 64, 32, [256, 1, 129], [700, 700, 385], seed=window % 1000, window=window)
    run(cache_dtype, 4, 1, 128, 8, [130, 1], [131, 500], seed=window % 1000, window=window, slopes=alibi(4))


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e2m1"])
@pytest.mark.parametrize("hd", [64, 128])
def test_windows_whose_rows_see_far_ahead(cache_dtype, hd):
    # many more keys than the window holds: they are split all the same, and none is left out
    for window in (1, 64):
        run(cache_dtype, 1, 1, hd, 16, [1500], [3000], seed=hd, window=window, hi=prefix(3000))
        run(cache_dtype, 2, 1, hd, 64, [20, 2], [2500, 1999], seed=hd, window=window, hi=prefix(2500), slopes=alibi(2) / 16)


@pytest.mark.parametrize("cache_dtype", ["bf16", "e2m1"])
def test_blocks_whose_tiles_see_different_keys(cache_dtype):
    # the first tile of 128 rows sees many keys, the second few or none, and the other way round
    n = 256
    p = torch.arange(n) + 400
    none = torch.full((n,), -1)
    for first, second in ((p, none), (none, p), (torch.full((n,), 600), torch.full((n,), 3)), (torch.full((n,), 3), p)):
        hi = torch.cat([first[:128], second[128:]])
        run(cache_dtype, 2, 2, 64, 16, [n], [n + 400], seed=3, hi=lambda lay: hi)
        run(cache_dtype, 2, 2, 128, 64, [n], [n + 400], seed=4, hi=lambda lay: hi, lo=lambda lay: hi - 200)
        run(cache_dtype, 2, 2, 128, 64, [n], [n + 400], seed=4, hi=lambda lay: hi, io="fp16")
    run(cache_dtype, 2, 2, 64, 16, [n], [n + 400], seed=3, hi=lambda lay: none)              # nobody sees anything
    run(cache_dtype, 2, 2, 64, 16, [5], [400], seed=3, lo=lambda lay: torch.full((5,), 10 ** 9))


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_caps_from_tiny_to_large(cache_dtype):
    for cap in (1e-20, 0.3, 15.0, 1000.0, 1e20):
        for new, length in (([1, 2], [100, 33]), ([80], [120])):
            run(cache_dtype, 2, 2, 64, 16, new, length, seed=2, cap=cap, q_gain=8.0)
            run(cache_dtype, 2, 2, 64, 16, new, length, seed=2, cap=cap, q_gain=8.0, scale=-0.2)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io", ["bf16", "fp16"])
def test_caps_against_scores_of_every_size(cache_dtype, io):
    # scores below a thousandth of the cap, around 0.3, 0.6 and 0.9 of it, and beyond; keys and queries far from 1, so that the unit of a product is too
    for q_gain, k_gain, scale in ((1.0, 1.0, 0.125), (1e3, 1e3, 1e-7), (1e-3, 1e-3, 1e5)):
        size = 5.0 * 8.0 * q_gain * k_gain * scale             # about the largest score of 80 rows and 120 keys of 64 elements
        for part in (1e-9, 1e-4, 0.3, 0.6, 0.9, 2.0):
            run(cache_dtype, 2, 2, 64, 16, [80, 1], [120, 50], seed=2, cap=size / part, q_gain=q_gain, k_gain=k_gain, scale=scale, io=io)


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_steep_slopes_over_far_keys(cache_dtype):
    # a mask that leaves only far keys: their differences count, not their distances
    slopes = torch.tensor([2.0, 0.01])
    for new in ([1], [64]):
        run(cache_dtype, 2, 2, 64, 16, new, [3000], seed=4, slopes=slopes, hi=lambda lay: torch.full((lay.n_tokens,), 40))
        run(cache_dtype, 2, 2, 64, 16, new, [3000], seed=4, slopes=-slopes, io="fp32" if cache_dtype == "fp32" else "bf16")


@pytest.mark.parametrize("cache_dtype", ["fp32", "bf16", "int8", "e2m1"])
def test_pages_that_do_not_exist_hide_their_keys(cache_dtype):
    for new, length in (([1, 2], [100, 40]), ([90, 1], [100, 40])):
        run(cache_dtype, 2, 2, 64, 16, new, length, seed=2, gone=((0, 1), (1, 0), (0, 5)), cap=10.0, window=60, slopes=alibi(2))


def test_queries_that_are_not_numbers_stay_in_their_rows():
    lay = P.Layout([1, 66], [40, 66], 16, seed=2)
    for cache_dtype in CACHES:
        cache = P.make_cache(lay, 2, 2, 64, cache_dtype)
        F.fill_any(cache, lay, seed=3)
        sc = binding.Scores(cap=5.0, slopes=alibi(2).cuda(), window=30)
        q = torch.randn(lay.n_tokens, 2, 64, generator=torch.Generator().manual_seed(4)).bfloat16()
        clean = cache.attention(0, q.cuda(), lay.batch(), scores=sc).cpu().double()
        q[0, 1, 3] = float("nan")
        q[20, 0, 5] = float("nan")
        got = cache.attention(0, q.cuda(), lay.batch(), scores=sc).cpu().double()
        assert bool(torch.isnan(got[0, 1]).all()) and bool(torch.isnan(got[20, 0]).all())
        got[0, 1], got[20, 0] = clean[0, 1], clean[20, 0]
        assert not bool(torch.isnan(got).any())
        assert float((got - clean).abs().max()) < 2.0 ** -7 * float(clean.abs().max())


def test_captured_calls_follow_the_masks():
    lay = P.Layout([1, 64, 3], [300, 120, 17], 16, seed=5, spare_columns=3)
    stream = torch.cuda.Stream()
    cache = P.make_cache(lay, 4, 4, 64, "bf16", stream=stream)
    contents = F.fill_any(cache, lay, seed=6)
    q = torch.randn(lay.n_tokens, 4, 64, generator=torch.Generator().manual_seed(7)).bfloat16()
    lo, hi, slopes = torch.zeros(lay.n_tokens, dtype=torch.int32).cuda(), torch.zeros(lay.n_tokens, dtype=torch.int32).cuda(), alibi(4).cuda()
    sc, batch, out, qd = binding.Scores(7.0, slopes, 100, lo, hi), lay.batch(max_len=0), torch.zeros_like(q).cuda(), q.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        cache.attention(0, qd, batch, out=out, scores=sc)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cache.attention(0, qd, batch, out=out, scores=sc)
    for seed in (8, 9):
        l, h = anything(seed, 100)(lay), anything(seed + 10, 200)(lay)
        lo.copy_(l)
        hi.copy_(h)
        slopes.copy_(alibi(4) * (seed - 7))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = S.reference(q, contents, lay, 0.125, 1, cap=7.0, slopes=slopes.cpu(), window=100, lo=l, hi=h)
        assert float(S.over(out.cpu(), *want, 64, q.dtype, 7.0).max()) <= 1
    assert cache.status() == 0


def test_refusals():
    lay = P.Layout([1, 2], [10, 20], 16)
    cache = P.make_cache(lay, 4, 2, 64, "bf16")
    q = torch.zeros(3, 4, 64, device="cuda")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in (dict(slopes=torch.zeros(3, device="cuda")), dict(lo=i32(2)), dict(hi=i32(4))):
        with pytest.raises(ValueError):
            cache.attention(0, q, lay.batch(), scores=binding.Scores(**bad))
    for bad in (dict(slopes=torch.zeros(4, device="cuda").double()), dict(lo=i32(3).long()), dict(hi=i32(6)[::2])):
        with pytest.raises(ValueError):
            binding.Scores(**bad)
    for bad in (dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-35), dict(window=-1)):
        with pytest.raises(binding.SdError) as e:
            cache.attention(0, q, lay.batch(), scores=binding.Scores(**bad))
        assert e.value.code == binding.SD_ERR_ARG
    import ctypes as C
    d = binding.SdHeads(q.data_ptr(), 256, 64, 0)
    assert binding.lib().sd_cache_attention_scores(cache.h, 0, lay.batch().ref, C.byref(d), 0.0, None, C.byref(d)) == binding.SD_ERR_ARG
    assert binding.lib().sd_cache_attention_scores(cache.h, 1, lay.batch().ref, C.byref(d), 0.0, C.byref(binding.SdScores()), C.byref(d)) == binding.SD_ERR_ARG
    assert cache.status() == 0


def test_wait_that_expires_is_reported():
    lay = P.Layout([300], [600], 32, seed=1)
    cache = P.make_cache(lay, 2, 2, 64, "bf16")
    contents = F.fill_any(cache, lay, seed=2)
    q = torch.randn(300, 2, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    sc = binding.Scores(cap=9.0)
    cache.set_option(binding.SD_CACHE_OPT_TEST_WAIT_EXPIRY, 1)
    cache.attention(0, q.cuda(), lay.batch(), scores=sc)
    assert cache.status() & binding.STATUS_WAIT_EXPIRED
    got = cache.attention(0, q.cuda(), lay.batch(), scores=sc).cpu()
    assert cache.status() == 0
    want = S.reference(q, contents, lay, 0.125, 1, cap=9.0)
    assert float(S.over(got, *want, 64, q.dtype, 9.0).max()) <= 1
