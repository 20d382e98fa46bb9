"""Attention of new tokens over a paged cache against the 64-bit form on the cache's own contents.

Tolerances.  With fp32 arithmetic a score is a sum of head_dim products in some order, off by at most (head_dim + 2) 2^-24 of
the sum of their magnitudes, plus 2^-22 for the scaling of q, the scales of an 8-bit cache and the base change; a weight's
exponential and the running rescalings cost at most 2^-19 (one 2^-22 step per key tile would be needed to pass it), sums of
up to 2^12 weights in a tree or in tiles 2^-19.  Queries and weights that enter the tensor cores as a high and a low 16-bit
part lose 2^-17 of themselves at most (bf16 parts; fp16 parts less).  Where they enter as one bf16, each product loses
2^-8 of itself and each weight 2^-8.
"""
import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


def rels(hd, cache_dtype, q_dtype, out_dtype):
    """(score_rel, weight_rel) of the arithmetic that the library documents for these types."""
    score, weight = (hd + 2 + 8) * 2.0 ** -24, 2.0 ** -18
    if cache_dtype != "fp32":
        score += 2.0 ** -16
        weight += 2.0 ** -16
        if out_dtype != torch.float32:                          # a 16-bit result may be computed with bf16 queries and weights
            score += 2.0 ** -8
            weight += 2.0 ** -8
    return score, weight


def run(cache_dtype, io, heads, kv_heads, hd, page, new, length, scale=None, out_dtype=None, seed=0, gain=1.0, **kw):
    lay = P.Layout(new, length, page, seed=seed, **kw)
    cache = P.make_cache(lay, heads, kv_heads, hd, cache_dtype)
    contents = P.fill(cache, lay, seed=seed + 1, k_gain=gain)
    g = torch.Generator().manual_seed(seed + 2)
    q = torch.randn(lay.n_tokens, heads, hd, generator=g).to(P.TORCH[io])
    out_dtype = P.TORCH[out_dtype or io]
    out = torch.full((lay.n_tokens, heads, hd), 9.0, dtype=out_dtype, device="cuda")
    cache.attention(0, q.cuda(), lay.batch(), scale=scale, out=out)
    assert cache.status() == 0
    cache.close()
    want, parts = P.attention(q, contents, lay, hd ** -0.5 if scale is None else scale, heads // kv_heads)
    lim = P.bound(want, parts, *rels(hd, cache_dtype, q.dtype, out_dtype), out_dtype)
    got = out.cpu().double()
    own = torch.zeros(lay.n_tokens, dtype=torch.bool)
    for s in range(len(new)):
        own[int(lay.first[s]):int(lay.first[s + 1])] = True
    assert bool((got[~own] == 9).all())                         # padding rows are left as they were
    err = ((got - want).abs() - lim)[own]
    assert not bool(torch.isnan(got).any())
    assert float(err.max()) <= 0, (float(err.max()), float((got - want)[own].abs().max()))


CACHES = ("fp32", "bf16", "int8", "e4m3")


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 64), (8, 2, 128), (3, 1, 32), (7, 1, 64), (12, 12, 128)])
def test_single_tokens(cache_dtype, heads, kv_heads, hd):
    run(cache_dtype, "fp32", heads, kv_heads, hd, 16, [1] * 7, [1, 2, 15, 16, 17, 100, 333], seed=heads)
    run(cache_dtype, "bf16", heads, kv_heads, hd, 8, [1, 0, 1], [9, 5, 64], seed=heads + 1, start=1, tail=2)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("io", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,hd,page", [(2, 2, 64, 16), (4, 1, 128, 64), (2, 1, 32, 8)])
def test_chunks(cache_dtype, io, heads, kv_heads, hd, page):
    # whole prompts, chunks after a prefix, single tokens, a sequence without new tokens and one shorter than its new tokens
    run(cache_dtype, io, heads, kv_heads, hd, page, [1, 33, 64, 130, 0, 5, 2], [70, 33, 65, 200, 40, 3, 0], seed=hd, tail=1)


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,length", [([128], [128]), ([127], [255]), ([129], [129]), ([256, 1], [513, 511]), ([300], [700]), ([1, 257], [1, 258])])
def test_chunk_borders(cache_dtype, hd, new, length):
    run(cache_dtype, "bf16", 2, 2, hd, 32, new, length, seed=sum(new))


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_long_sequences(cache_dtype):
    run(cache_dtype, "fp32", 4, 2, 64, 64, [1, 1], [4001, 63], seed=5)
    run(cache_dtype, "bf16", 8, 1, 128, 128, [2], [2500], seed=6)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
def test_page_lengths(cache_dtype, page):
    run(cache_dtype, "bf16", 2, 2, 64, page, [1, 40], [page * 3 + 1, 150], seed=page)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("scale,gain", [(0.05, 1.0), (-0.3, 1.0), (1.0, 4.0), (None, 1e-6), (1e-7, 1e6)])
def test_scales_and_magnitudes(cache_dtype, scale, gain):
    # scores from nearly equal to dominated by one key; keys of tiny and of large magnitude
    run(cache_dtype, "fp32", 2, 1, 64, 16, [1, 20], [50, 64], scale=scale, gain=gain, seed=11)


@pytest.mark.parametrize("io,out", [("fp32", "fp16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp16", "bf16")])
@pytest.mark.parametrize("cache_dtype", CACHES)
def test_output_types(cache_dtype, io, out):
    run(cache_dtype, io, 2, 2, 64, 16, [1, 70], [30, 100], out_dtype=out, seed=21)


def test_scales_of_very_different_sizes():
    # values whose scales differ by 2^60 between neighbouring tokens, and tokens whose values are all zero
    lay = P.Layout([1, 1], [77, 16], 16, seed=3)
    cache = P.make_cache(lay, 2, 2, 64, "int8")
    contents = P.fill(cache, lay, seed=4)
    pool = cache.layer(0)
    for s, l in enumerate(lay.length):
        for p in range(l):
            page, slot = lay.slot(s, p)
            f = 0.0 if (p % 5 == 0 or s == 1) else 2.0 ** (12 * (p % 6) - 30)
            pool["v_scale"][page, :, slot] *= f
            contents[s][1][:, p] *= f
    q = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(1))
    got = cache.attention(0, q.cuda(), lay.batch()).cpu().double()
    want, parts = P.attention(q, contents, lay, 0.125, 1)
    lim = P.bound(want, parts, *rels(64, "int8", torch.float32, torch.float32), torch.float32)
    assert bool(((got - want).abs() <= lim).all())
    assert bool((got[1] == 0).all())
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8"])
def test_strided_queries_and_outputs(cache_dtype):
    lay = P.Layout([3, 1, 70], [30, 17, 90], 16, seed=8)
    H, hd, n = 4, 64, 74
    cache = P.make_cache(lay, H, H, hd, cache_dtype)
    contents = P.fill(cache, lay, seed=9)
    g = torch.Generator().manual_seed(10)
    for make in (lambda: torch.randn(n, 3 * H * hd, generator=g)[:, :H * hd].unflatten(1, (H, hd)),
                 lambda: torch.randn(n, H, hd + 3, generator=g)[..., 3:],
                 lambda: torch.randn(H, n, hd, generator=g).transpose(0, 1),
                 lambda: torch.randn(n, 1, hd, generator=g).expand(n, H, hd)):
        q = make()
        dev = torch.empty_strided(q.shape, q.stride(), device="cuda") if q.stride(1) else q[:, :1].cuda().expand(n, H, hd)
        if q.stride(1):
            dev.copy_(q)
        out = torch.zeros(H, n, hd + 1, device="cuda").transpose(0, 1)[..., 1:]
        cache.attention(0, dev, lay.batch(), out=out)
        want, parts = P.attention(q, contents, lay, hd ** -0.5, 1)
        lim = P.bound(want, parts, *rels(hd, cache_dtype, torch.float32, torch.float32), torch.float32)
        assert bool(((out.cpu().double() - want).abs() <= lim).all())
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_bad_pages_are_masked_and_reported(cache_dtype):
    # the keys of a page that does not exist are left out of the sums; a row that has no other keys is zero
    lay = P.Layout([1, 1, 20], [40, 10, 40], 16, seed=2)
    cache = P.make_cache(lay, 2, 2, 64, cache_dtype)
    contents = P.fill(cache, lay, seed=3)
    q = torch.randn(22, 2, 64, generator=torch.Generator().manual_seed(1))
    pages = lay.pages.clone()
    pages[0, 1], pages[1, 0], pages[2, 0] = lay.n_pages, -1, 1 << 30
    out = cache.attention(0, q.cuda(), binding.CacheBatch(pages.cuda(), lay.first.cuda(), lay.len.cuda(), 22, 20)).cpu().double()
    assert cache.status() == binding.STATUS_BAD_BATCH
    keep = [torch.arange(40) // 16 != 1, torch.zeros(10, dtype=torch.bool), torch.arange(40) >= 16]
    score_rel, weight_rel = rels(64, cache_dtype, torch.float32, torch.float32)
    for r, s, p in lay.places():
        k, v = contents[s]
        seen = keep[s] & (torch.arange(len(keep[s])) <= p)
        if not bool(seen.any()):
            assert bool((out[r] == 0).all())
            continue
        w = torch.softmax(torch.einsum("hd,hjd->hj", q[r].double(), k[:, seen]) * 0.125, -1)
        want = torch.einsum("hj,hjd->hd", w, v[:, seen])
        assert float((out[r] - want).abs().max()) <= 40 * (score_rel + weight_rel)      # terms stay below 10, values below 5
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
def test_steps_replayed_from_a_graph(cache_dtype):
    # append + attention captured once, replayed with other lengths, pages and inputs in the same device arrays
    H, hd, page, steps = 4, 64, 16, 24
    lay = P.Layout([1, 1], [30 + steps, 5 + steps], page, seed=1)
    cache = P.make_cache(lay, H, H, hd, cache_dtype)
    eager = P.make_cache(lay, H, H, hd, cache_dtype)
    for c in (cache, eager):
        P.fill(c, lay, seed=2)
    length = torch.tensor([30, 5], dtype=torch.int32, device="cuda")
    b = binding.CacheBatch(lay.pages.cuda(), lay.first.cuda(), length, 2, 1, max(lay.length))
    q, k, v = (torch.zeros(2, H, hd, device="cuda") for _ in range(3))
    out = torch.zeros(2, H, hd, device="cuda")
    eager.append(0, k, v, b)                                    # the warm-up below writes the same place of the other cache
    torch.cuda.synchronize()
    with torch.cuda.stream(cache.stream):
        cache.append(0, k, v, b)
        cache.attention(0, q, b, out=out)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=cache.stream):
            cache.append(0, k, v, b)
            cache.attention(0, q, b, out=out)
    g = torch.Generator().manual_seed(7)
    for t in range(steps):
        for x in (q, k, v):
            x.copy_(torch.randn(2, H, hd, generator=g))
        length += 1
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager.append(0, k, v, b)
        want = eager.attention(0, q, b)
        assert torch.equal(got, want), t
    for n, t in cache.layer(0).items():
        assert torch.equal(t.view(torch.uint8), eager.layer(0)[n].view(torch.uint8))
    assert cache.status() == 0 and eager.status() == 0
    cache.close()
    eager.close()


def test_another_stream_and_two_caches_at_once():
    lay = P.Layout([1, 50], [600, 130], 16, seed=6)
    caches = [P.make_cache(lay, 4, 2, 64, "int8") for _ in range(2)]
    contents = [P.fill(c, lay, seed=s) for s, c in enumerate(caches)]
    q = torch.randn(51, 4, 64, generator=torch.Generator().manual_seed(1))
    side = torch.cuda.Stream()
    outs = []
    with torch.cuda.stream(side):
        dev = q.cuda()
        b = lay.batch()
        for _ in range(20):                                     # both in flight together, inputs and outputs from a third stream
            outs = [c.attention(0, dev * 1.0, b) for c in caches]
        outs = [o * 1.0 for o in outs]
    side.synchronize()
    for o, con in zip(outs, contents):
        want, parts = P.attention(q, con, lay, 0.125, 2)
        lim = P.bound(want, parts, *rels(64, "int8", torch.float32, torch.float32), torch.float32)
        assert bool(((o.cpu().double() - want).abs() <= lim).all())
    for c in caches:
        c.close()


def test_same_call_twice_gives_the_same_bits():
    for cache_dtype in CACHES:
        lay = P.Layout([1, 90, 1], [3000, 200, 5], 32, seed=6)
        cache = P.make_cache(lay, 4, 2, 128, cache_dtype)
        P.fill(cache, lay)
        q = torch.randn(92, 4, 128, generator=torch.Generator().manual_seed(1)).cuda()
        one = cache.attention(0, q, lay.batch())
        for _ in range(5):
            assert torch.equal(one, cache.attention(0, q, lay.batch()))
        cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd,page", [(64, 16), (128, 8), (128, 64)])
def test_many_runs_of_a_mixed_batch_agree(cache_dtype, hd, page):
    # blocks of every length side by side, two hundred times: a result that is read before its last product shows here
    new, length = [1, 33, 64, 130, 0, 5, 2, 300, 256, 129], [70, 33, 65, 200, 40, 3, 0, 900, 1024, 3000]
    lay = P.Layout(new, length, page, seed=1)
    cache = P.make_cache(lay, 4, 1, hd, cache_dtype)
    contents = P.fill(cache, lay, seed=2)
    q = torch.randn(lay.n_tokens, 4, hd, generator=torch.Generator().manual_seed(3)).bfloat16()
    dev, b = q.cuda(), lay.batch()
    one = cache.attention(0, dev, b)
    want, parts = P.attention(q, contents, lay, hd ** -0.5, 4)
    lim = P.bound(want, parts, *rels(hd, cache_dtype, torch.bfloat16, torch.bfloat16), torch.bfloat16)
    assert bool(((one.cpu().double() - want).abs() <= lim).all())
    out = torch.empty_like(one)
    for _ in range(20 if cache_dtype == "fp32" else 200):
        assert torch.equal(cache.attention(0, dev, b, out=out), one)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype,hd", [("bf16", 128), ("e4m3", 64)])
def test_no_wait_runs_out_when_the_gpu_is_full(cache_dtype, hd):
    # more blocks than processors and several heads, a hundred times: a wait for a phase that has been passed shows as a bad status
    new = [40 + (37 * i) % 290 for i in range(32)]
    lay = P.Layout(new, [n + (211 * i) % 1200 for i, n in enumerate(new)], 32, seed=4)
    cache = P.make_cache(lay, 8, 4, hd, cache_dtype)
    P.fill(cache, lay, seed=5)
    dev, b = torch.randn(lay.n_tokens, 8, hd, generator=torch.Generator().manual_seed(6)).bfloat16().cuda(), lay.batch()
    one = cache.attention(0, dev, b)
    out = torch.empty_like(one)
    for _ in range(100):
        assert torch.equal(cache.attention(0, dev, b, out=out), one)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("hd,heads,page", [(64, 4, 16), (128, 7, 64)])
def test_chunks_whose_keys_are_split(cache_dtype, hd, heads, page):
    # few query rows over long sequences: keys split over blocks, rows that see fewer keys than others, a sequence that sees none of the
    # later splits, and rows without a place
    run(cache_dtype, "bf16", heads, 1, hd, page, [100, 40, 300, 9], [2900, 2049, 300, 4], seed=hd, start=2, tail=1)
    run(cache_dtype, "bf16", heads, 1, hd, page, [65], [3333], seed=hd + 1)


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(2, 2, 64), (12, 1, 128), (24, 1, 64), (25, 1, 64), (64, 2, 128)])
def test_numbers_of_rows_at_which_the_kernel_changes(cache_dtype, heads, kv_heads, hd):
    group = heads // kv_heads
    run(cache_dtype, "bf16", heads, kv_heads, hd, 16, [-(-n // group) for n in (8, 9, 16, 17, 24, 25, 32, 33)], [40, 50, 60, 17, 300, 25, 33, 900], seed=heads)
    run(cache_dtype, "bf16", heads, kv_heads, hd, 16, [1, 1, 1], [1, 700, 64], seed=heads + 1)


@pytest.mark.parametrize("cache_dtype", ["bf16", "e4m3"])
def test_the_length_hint_only_splits(cache_dtype):
    lay = P.Layout([70, 1, 50], [2600, 2000, 1100], 32, seed=1)
    cache = P.make_cache(lay, 4, 1, 64, cache_dtype)
    contents = P.fill(cache, lay, seed=2)
    q = torch.randn(lay.n_tokens, 4, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    want, parts = P.attention(q, contents, lay, 0.125, 4)
    lim = P.bound(want, parts, *rels(64, cache_dtype, q.dtype, q.dtype), q.dtype)
    for hint in (0, 1, 1024, 2600, 1 << 30):                    # unknown, far too short, too short, right, far too long
        b = lay.batch(max_len=hint)
        one = cache.attention(0, q.cuda(), b)
        assert bool(((one.cpu().double() - want).abs() <= lim).all()), hint
        for _ in range(20):
            assert torch.equal(cache.attention(0, q.cuda(), b), one)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("new,length", [([1, 1], [70, 3]), ([50, 1], [60, 9]), ([40, 2], [2100, 2]), ([1], [3000])])
def test_a_query_that_is_not_a_number_spoils_its_own_row_only(cache_dtype, new, length):
    lay = P.Layout(new, length, 16, seed=7)
    cache = P.make_cache(lay, 2, 2, 64, cache_dtype)
    contents = P.fill(cache, lay, seed=8)
    q = torch.randn(lay.n_tokens, 2, 64, generator=torch.Generator().manual_seed(9)).bfloat16()
    want, parts = P.attention(q, contents, lay, 0.125, 1)
    lim = P.bound(want, parts, *rels(64, cache_dtype, q.dtype, q.dtype), q.dtype)
    q[0, 1, 5] = float("nan")
    got = cache.attention(0, q.cuda(), lay.batch()).cpu().double()
    assert bool(torch.isnan(got[0, 1]).all())
    got[0, 1] = want[0, 1]
    assert bool(((got - want).abs() <= lim).all())
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8"])
@pytest.mark.parametrize("new", [[1, 1], [140, 33]])
def test_pages_past_32_bits_of_elements_and_shared_pages(cache_dtype, new):
    # the same contents in the first pages of a small cache and in the last of a pool with more than 2^32 elements; there the
    # second sequence's first page is the first sequence's
    heads, kv, hd, page = 8, 8, 128, 128
    many = (1 << 32) // (kv * page * hd) + 40
    length = [300, 260]
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(sum(length), kv, hd, generator=g).bfloat16() for _ in range(2))
    k[300:300 + page], v[300:300 + page] = k[:page], v[:page]
    q = torch.randn(sum(new), heads, hd, generator=g).bfloat16().cuda()
    out = []
    for n_pages, table in ((6, [[0, 1, 2], [3, 4, 5]]), (many, [[many - 1, many - 9, many - 2], [many - 1, many - 30, many - 5]])):
        cache = binding.PagedCache(1, heads, kv, hd, page, n_pages, 4, 600, dtype=cache_dtype)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        for s in range(2):                                         # one sequence per call: the shared page is written twice, alike
            rows = slice(0, 300) if s == 0 else slice(300, 560)
            b = binding.CacheBatch(i32([table[s]]), i32([0, length[s]]), i32([length[s]]), length[s], length[s])
            cache.append(0, k[rows].cuda(), v[rows].cuda(), b)
            rk, rv = cache.read(0, b)
            assert torch.equal(rk.cpu(), P.stored(k[rows].float(), cache_dtype)) and torch.equal(rv.cpu(), P.stored(v[rows].float(), cache_dtype))
        b = binding.CacheBatch(i32(table), i32([0, new[0], sum(new)]), i32(length), sum(new), max(new), max(length))
        out.append(cache.attention(0, q, b))
        assert cache.status() == 0
        cache.close()
        del cache
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("graphed", [False, True])
@pytest.mark.parametrize("new", [[300] * 12, [300, 1] * 6])
def test_what_follows_on_the_stream_sees_all_results(graphed, new):
    # the second launch of a call may begin, and have nothing to do, before the first has ended; a copy queued right behind it waits for both
    lay = P.Layout(new, [900] * 12, 32, seed=1)
    cache = P.make_cache(lay, 16, 16, 64, "bf16")
    P.fill(cache, lay, seed=2)
    q = torch.randn(lay.n_tokens, 16, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    b = lay.batch()
    want = cache.attention(0, q, b).clone()
    out, copy = torch.empty_like(want), torch.empty_like(want)
    torch.cuda.synchronize()

    def step():
        out.zero_()
        cache.attention(0, q, b, out=out)
        copy.copy_(out)

    with torch.cuda.stream(cache.stream):
        if graphed:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=cache.stream):
                step()
        for _ in range(100):
            copy.zero_()
            graph.replay() if graphed else step()
            assert torch.equal(copy, want)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8"])
def test_threads_may_share_a_cache(cache_dtype):
    # calls of two launches that pass shares of split keys on through the cache's workspace: they must stay together
    import threading
    lay = P.Layout([70, 1], [2600, 900], 32, seed=1)
    cache = P.make_cache(lay, 4, 1, 64, cache_dtype)
    P.fill(cache, lay, seed=2)
    g = torch.Generator().manual_seed(3)
    b = lay.batch()
    queries = [torch.randn(lay.n_tokens, 4, 64, generator=g).bfloat16().cuda() for _ in range(4)]
    want = [cache.attention(0, q, b) for q in queries]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(cache.stream):
            out = torch.empty_like(want[i])
            for _ in range(100):
                cache.attention(0, queries[i], b, out=out)
                if not torch.equal(out, want[i]):
                    wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    assert cache.status() == 0
    cache.close()


def two_keys(cache_dtype, hd, q, k, v, scale):
    """Attention of single tokens over two keys each: q [seqs, heads, hd], k and v [2, hd] alike for all."""
    seqs, heads = q.shape[:2]
    cache = binding.PagedCache(1, heads, heads, hd, 8, seqs, seqs, 2 * seqs, dtype=cache_dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages, length = i32([[s] for s in range(seqs)]), i32([2] * seqs)
    both = binding.CacheBatch(pages, i32([2 * s for s in range(seqs + 1)]), length, 2 * seqs, 2, 2)
    rows = lambda x: x.unsqueeze(1).expand(2, heads, hd).repeat(seqs, 1, 1).cuda()  # noqa: E731
    cache.append(0, rows(k), rows(v), both)
    out = cache.attention(0, q.cuda(), binding.CacheBatch(pages, i32(list(range(seqs + 1))), length, seqs, 1, 2), scale=scale).cpu().double()
    assert out.dtype == torch.float64 and cache.status() == 0
    cache.close()
    return out


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_fp32_results_keep_the_bits_of_fp32_queries(cache_dtype, hd):
    # Scores 0 and -hd scale q with q = 1 + 2^-9 + 2^-18 in every element: the sums are exact in fp32, and parts of 8 + 8 bits would lose the
    # last term.  The result is the second key's weight e^-10: the exponent of size 14.4 in base 2 is rounded three times (the scale in base 2, the
    # product, the subtraction), 3 * 14.4 * 2^-24 * ln 2 = 1.8e-6, the key's scale in 8 bits and a query of 22 bits cost as much again,
    # the exponential 2^-22, weights and division 2^-22 each: below 2^-17.  Without the last term it would be 10 * 2^-18 off.
    # In 8 bits small weights lie on a fixed grid, each off by up to 2^-32 of the largest value (see paged_reference.bound): two keys, 2^-31.
    q = torch.full((3, 5, hd), 1 + 2.0 ** -9 + 2.0 ** -18)
    scale = float(torch.tensor(10.0 / hd))
    k, v = torch.stack([torch.zeros(hd), -torch.ones(hd)]), torch.stack([torch.zeros(hd), torch.ones(hd)])
    got = two_keys(cache_dtype, hd, q, k, v, scale)
    s = -hd * scale * (1 + 2.0 ** -9 + 2.0 ** -18)
    want = torch.exp(torch.tensor(s, dtype=torch.float64)) / (1 + torch.exp(torch.tensor(s, dtype=torch.float64)))
    assert float((got - want).abs().max()) <= want * 2.0 ** -17 + (2.0 ** -31 if cache_dtype in P.TOP else 0)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_fp32_results_keep_the_bits_of_the_weights(cache_dtype, hd):
    # Values 1 and -1 under nearly equal weights 1 and p = e^-s, s from 0.005 to 0.02: the result (1 - p) / (1 + p) is s / 2, and an error of p
    # moves it by half of that error.  The exponential is off by 2^-22 at most, p as two parts of 11 or three of 8 bits by 2^-22, the sums of numbers
    # near 1 by 2^-23, the exponent (below 2^-5) by less than 2^-27: 2^-21 in all.  Two parts of 8 bits would lose up to 2^-17.
    g = torch.Generator().manual_seed(3)
    q = torch.zeros(8, 16, hd)
    q[..., 0] = 0.005 + 0.015 * torch.rand(8, 16, generator=g)
    k = torch.zeros(2, hd)
    k[1, 0] = -1.0
    v = torch.stack([torch.ones(hd), -torch.ones(hd)])
    got = two_keys(cache_dtype, hd, q, k, v, 1.0)
    want = torch.tanh(q[..., :1].double() / 2)
    assert float((got - want).abs().max()) <= 2.0 ** -21
