"""Attention of chunks over a paged cache, held to a limit that one missing key exceeds (see paged_bounds): the kernel for many query
rows, its split keys, masks, missing pages, scales and both ways in which pages reach it."""
import pytest
import torch

import paged_bounds as B
import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu

CACHES = ("bf16", "int8", "e4m3")


def run(cache_dtype, heads, kv_heads, hd, page, new, length, scale=None, seed=0, io="bf16", out_dtype=None, gone=(), max_new=None, max_len=None, k_gain=1.0, **kw):
    """gone: (sequence, column) of table entries that are made to name no page."""
    lay = P.Layout(new, length, page, seed=seed, **kw)
    cache = P.make_cache(lay, heads, kv_heads, hd, cache_dtype)
    contents = P.fill(cache, lay, seed=seed + 1, k_gain=k_gain)
    q = torch.randn(lay.n_tokens, heads, hd, generator=torch.Generator().manual_seed(seed + 2)).to(P.TORCH[io])
    pages, exists = lay.pages.clone(), [torch.ones(l, dtype=torch.bool) for l in length]
    for i, (s, column) in enumerate(gone):
        pages[s, column] = (-1, lay.n_pages, 1 << 30)[i % 3]
        exists[s][column * page:(column + 1) * page] = False
    b = binding.CacheBatch(pages.cuda(), lay.first.cuda(), lay.len.cuda(), lay.n_tokens, max_new or max(new), max(length) if max_len is None else max_len)
    out = torch.full(q.shape, 9.0, dtype=P.TORCH[out_dtype or io], device="cuda")
    cache.attention(0, q.cuda(), b, scale=scale, out=out)
    status = cache.status()
    again = torch.full_like(out, 9.0)
    cache.attention(0, q.cuda(), b, scale=scale, out=again)
    assert torch.equal(out, again)
    cache.close()
    assert status == (binding.STATUS_BAD_BATCH if gone else 0)
    want, R, terms = B.reference(q, contents, lay, hd ** -0.5 if scale is None else scale, heads // kv_heads, exists)
    own = torch.zeros(lay.n_tokens, dtype=torch.bool)
    for s in range(len(new)):
        own[int(lay.first[s]):int(lay.first[s + 1])] = True
    got = out.cpu()
    assert bool((got[~own] == 9).all())
    over = B.over(got, want, R, terms, hd, q.dtype)[own]
    assert not bool(torch.isnan(over).any())
    assert float(over.max()) <= 1, (float(over.max()), float(over.median()), int(over.argmax()))


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd,heads,page", [(64, 4, 16), (64, 4, 128), (128, 7, 64), (128, 4, 8)])
def test_split_keys(cache_dtype, hd, heads, page):
    run(cache_dtype, heads, 1, hd, page, [100, 40, 300, 9], [2900, 2049, 300, 4], seed=hd, start=2, tail=1)
    run(cache_dtype, heads, 1, hd, page, [65], [3333], seed=hd + 1)
    run(cache_dtype, heads, 1, hd, page, [33, 8], [4097, 2560], seed=hd + 2, max_len=1500)      # longer than the hint: the last split takes the rest


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,length", [([128], [128]), ([127], [255]), ([129], [129]), ([256, 1], [513, 511]), ([300], [700]), ([64, 257], [64, 258]),
                                         ([65, 130, 191], [193, 320, 191])])
def test_borders_of_tiles(cache_dtype, hd, new, length):
    for page in (8, 32, 128):
        run(cache_dtype, 2, 2, hd, page, new, length, seed=sum(new) + page)


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_chunks_beside_single_tokens(cache_dtype):
    run(cache_dtype, 8, 4, 64, 16, [1] * 20 + [200] + [1] * 3 + [40, 0], [17 * i + 1 for i in range(20)] + [700, 1, 1000, 64, 41, 5], seed=3)
    run(cache_dtype, 8, 2, 128, 32, [1, 150, 1], [2500, 190, 33], seed=4, tail=2)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (4, 4), (7, 1)])
def test_long_single_tokens_beside_a_chunk_are_split_too(cache_dtype, heads, kv_heads):
    # the chunk's rows take none of the workspace of the few rows' partial results: all their splits are joined beside it
    run(cache_dtype, heads, kv_heads, 128, 64, [1, 512, 1, 2, 8], [9000, 700, 20, 7777, 5001], seed=13)
    run(cache_dtype, heads, kv_heads, 64, 16, [1, 1030, 3], [20001, 1030, 6000], seed=14, start=1, tail=3)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [64, 128])
def test_one_sequence_of_few_rows_under_a_larger_bound(cache_dtype, hd):
    run(cache_dtype, 2, 2, hd, 16, [3], [700], seed=5, tail=60, max_new=60)
    run(cache_dtype, 2, 2, hd, 16, [1], [3001], seed=6, tail=60, max_new=60)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("scale,k_gain", [(0.05, 1.0), (-0.3, 1.0), (-0.02, 3.0), (1.0, 0.5), (1e-7, 1e6), (3e4, 1e-6)])
def test_scales(cache_dtype, hd, io, scale, k_gain):
    run(cache_dtype, 2, 1, hd, 16, [40, 70, 1], [50, 300, 90], scale=scale, k_gain=k_gain, seed=11, io=io)
    run(cache_dtype, 2, 1, hd, 64, [60], [2100], scale=scale, k_gain=k_gain, seed=12, io=io)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 64, 128])
def test_pages_that_do_not_exist(cache_dtype, hd, page):
    # in the first tile, between whole tiles, a whole tile, the one that holds a row's own key; nothing left for the first rows
    n = 700 // page
    run(cache_dtype, 2, 2, hd, page, [50, 60], [700, 90], gone=[(0, 0), (0, n // 2), (0, n)], seed=page)
    run(cache_dtype, 2, 2, hd, page, [130], [700], gone=[(0, c) for c in range(128 // page, 256 // page)] + [(0, n)], seed=page + 1)
    run(cache_dtype, 2, 2, hd, page, [150, 150], [150, 150], gone=[(0, c) for c in range(1 + 64 // page)] + [(1, 1)], seed=page + 2)
    run(cache_dtype, 2, 2, hd, page, [40], [3000], gone=[(0, 1000 // page), (0, 2999 // page)], seed=page + 3)      # split keys


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io,out", [("fp16", "fp16"), ("fp32", "fp16"), ("fp32", "bf16"), ("fp16", "bf16"), ("bf16", "fp16")])
@pytest.mark.parametrize("hd,heads,kv_heads,page", [(64, 4, 2, 16), (128, 3, 3, 64)])
def test_types_that_keep_more_than_bf16(cache_dtype, io, out, hd, heads, kv_heads, page):
    # queries or results with more bits than a bf16: queries and weights enter with 16 bits
    run(cache_dtype, heads, kv_heads, hd, page, [1, 33, 140, 300, 5], [70, 600, 150, 900, 3], io=io, out_dtype=out, seed=hd, start=1, tail=2)
    run(cache_dtype, heads, kv_heads, hd, page, [70], [2500], io=io, out_dtype=out, seed=hd + 1)                   # split keys
    run(cache_dtype, heads, kv_heads, hd, page, [129, 128, 127], [129, 400, 255], io=io, out_dtype=out, scale=-0.5, seed=hd + 2)
    run(cache_dtype, heads, kv_heads, hd, page, [60, 61], [700, 130], io=io, out_dtype=out, seed=hd + 3, gone=[(0, 0), (0, 200 // page), (1, 128 // page)])


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("new,length,page,heads", [([300], [1000], 64, 80), ([50, 1], [13000, 5], 16, 2), ([200, 50], [900, 820], 8, 80)])
def test_a_wait_that_runs_out_is_reported_and_the_cache_stays_usable(cache_dtype, io, new, length, page, heads):
    # the loaders give up with tensor copies (bf16) of a tile's keys on their way; they end with the copies, not with a time limit.  As many
    # heads, or positions, as leave a block more tiles of keys than it has stages
    import time
    lay = P.Layout(new, length, page, seed=9)
    cache = P.make_cache(lay, heads, heads, 128, cache_dtype)
    P.fill(cache, lay, seed=10)
    q = torch.randn(lay.n_tokens, heads, 128, generator=torch.Generator().manual_seed(11)).to(P.TORCH[io]).cuda()
    b = lay.batch()
    want = cache.attention(0, q, b)
    assert cache.status() == 0
    for value in (2, -1):
        with pytest.raises(binding.SdError):
            cache.set_option(binding.SD_CACHE_OPT_TEST_WAIT_EXPIRY, value)
    with pytest.raises(binding.SdError):
        cache.set_option(99, 1)
    for _ in range(3):
        cache.set_option(binding.SD_CACHE_OPT_TEST_WAIT_EXPIRY, 1)
        t0 = time.perf_counter()
        cache.attention(0, q, b)
        assert cache.status() == binding.STATUS_WAIT_EXPIRED
        assert time.perf_counter() - t0 < 0.5                   # a millisecond or two; the limit of a wait is two seconds
        assert torch.equal(cache.attention(0, q, b), want)
        assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("new,length", [([3, 1, 70], [30, 17, 90]), ([74], [1500])])
def test_strided_queries_and_outputs(cache_dtype, io, new, length):
    # slices of wider rows, nothing 16-byte aligned, heads ahead of rows, one query for all heads; results into a strided tensor
    lay = P.Layout(new, length, 16, seed=8)
    H, hd, n = 4, 64, 74
    cache = P.make_cache(lay, H, H, hd, cache_dtype)
    contents = P.fill(cache, lay, seed=9)
    g = torch.Generator().manual_seed(10)
    draw = lambda *shape: torch.randn(*shape, generator=g).to(P.TORCH[io]).cuda()  # noqa: E731
    for q in (draw(n, 3 * H * hd)[:, :H * hd].unflatten(1, (H, hd)), draw(n, H, hd + 3)[..., 3:], draw(H, n, hd).transpose(0, 1), draw(n, 1, hd).expand(n, H, hd)):
        wide = torch.full((H, n, hd + 1), 5.0, dtype=q.dtype, device="cuda")
        out = wide.transpose(0, 1)[..., 1:]
        cache.attention(0, q, lay.batch(), out=out)
        want, R, terms = B.reference(q.cpu(), contents, lay, hd ** -0.5, 1)
        assert float(B.over(out.cpu(), want, R, terms, hd, q.dtype).max()) <= 1
        assert bool((wide[..., 0] == 5).all())
        assert torch.equal(out, cache.attention(0, q, lay.batch()))
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("new,length", [([50, 60, 1], [60, 200, 9]), ([70], [3000])])
def test_a_query_that_is_not_finite_spoils_its_own_row_only(cache_dtype, new, length):
    lay = P.Layout(new, length, 16, seed=7)
    cache = P.make_cache(lay, 2, 2, 64, cache_dtype)
    contents = P.fill(cache, lay, seed=8)
    q = torch.randn(lay.n_tokens, 2, 64, generator=torch.Generator().manual_seed(9)).half()
    ref = B.reference(q, contents, lay, 0.125, 1)
    for value in (float("nan"), float("inf"), float("-inf")):
        bad = q.clone()
        bad[7, 1, 5] = value
        got = cache.attention(0, bad.cuda(), lay.batch()).cpu()
        assert bool((torch.isnan(got[7, 1]) | ((got[7, 1] == 0) & (value == value))).all())
        got[7, 1] = ref[0][7, 1].half()
        assert float(B.over(got, *ref, 64, q.dtype).max()) <= 1
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("new,length", [([300] * 4, [900] * 4), ([300, 1] * 3, [900, 2000] * 3), ([64], [4000])])
def test_captured_calls_with_pairs(cache_dtype, new, length):
    # one graph replayed with other queries in the same memory, a copy right behind each call
    lay = P.Layout(new, length, 32, seed=1)
    cache = P.make_cache(lay, 4, 2, 128, cache_dtype)
    P.fill(cache, lay, seed=2)
    b = lay.batch()
    q = torch.zeros(lay.n_tokens, 4, 128, dtype=torch.float16, device="cuda")
    out, copy = torch.zeros_like(q), torch.zeros_like(q)
    with torch.cuda.stream(cache.stream):
        cache.attention(0, q, b, out=out)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=cache.stream):
            cache.attention(0, q, b, out=out)
            copy.copy_(out)
        g = torch.Generator(device="cuda").manual_seed(3)
        for _ in range(20):
            q.normal_(generator=g)
            graph.replay()
            got = copy.clone()
            assert torch.equal(got, cache.attention(0, q, b))
    assert cache.status() == 0
    cache.close()
