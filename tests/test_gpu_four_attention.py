"""Attention over a paged cache in 4 bits, and a model on it, against the 64-bit form on the cache's own contents.

Tolerances are those of the 8-bit caches, whose arithmetic this is (a code times its block scale is a 16-bit number exactly): scores
(head_dim + 10) 2^-24 + 2^-16 of the sum of their terms' magnitudes, weights 2^-18 + 2^-16, and 2^-8 more of each where
the result has 16 bits.  The smallest weights lie on fp16's grid: per key 2^-31 of the largest |value| (2^-25 of a unit times a value of up to
2688 scales, the unit at most twice the largest scale over 2^7).
"""
import pytest
import torch

import four_reference as F
import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


def limit(want, parts, hd, out_dtype, fine=False):
    """fine: queries and weights as two fp16.  A query's element is off by 2^-22 of itself or 2^-25 of the row's largest, which is 2^-20 of a score's terms
    while the largest times the sum of the keys' magnitudes is at most 2^4 times theirs; a weight by 2^-22."""
    more = 0.0 if out_dtype == torch.float32 else 2.0 ** -8
    pair = 2.0 ** -20 if fine else 2.0 ** -16
    lim = P.bound(want, parts, (hd + 10) * 2.0 ** -24 + pair + more, 2.0 ** -18 + pair + more, out_dtype)
    return lim + parts[2].unsqueeze(-1) * 2.0 ** -31


def run(io, heads, kv_heads, hd, page, new, length, scale=None, out_dtype=None, seed=0, k_gain=1.0, v_gain=1.0, max_len=None, fine=False, **kw):
    lay = P.Layout(new, length, page, seed=seed, **kw)
    cache = P.make_cache(lay, heads, kv_heads, hd, "e2m1")
    contents = F.fill(cache, lay, seed=seed + 1, k_gain=k_gain, v_gain=v_gain)
    q = torch.randn(lay.n_tokens, heads, hd, generator=torch.Generator().manual_seed(seed + 2)).to(P.TORCH[io])
    out_dtype = P.TORCH[out_dtype or io]
    out = torch.full((lay.n_tokens, heads, hd), 9.0, dtype=out_dtype, device="cuda")
    cache.attention(0, q.cuda(), lay.batch(max_len=max_len), scale=scale, out=out)
    assert cache.status() == 0
    cache.close()
    want, parts = P.attention(q, contents, lay, hd ** -0.5 if scale is None else scale, heads // kv_heads)
    got = out.cpu().double()
    own = torch.zeros(lay.n_tokens, dtype=torch.bool)
    for s in range(len(new)):
        own[int(lay.first[s]):int(lay.first[s + 1])] = True
    assert bool((got[~own] == 9).all())                         # padding rows are left as they were
    assert not bool(torch.isnan(got).any())
    err = ((got - want).abs() - limit(want, parts, hd, out_dtype, fine))[own]
    assert float(err.max()) <= 0, (float(err.max()), float((got - want)[own].abs().max()))
    return got, want


@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 64), (8, 2, 128), (3, 1, 32), (7, 1, 64), (12, 12, 128), (2, 2, 32)])
def test_single_tokens(heads, kv_heads, hd):
    run("fp32", heads, kv_heads, hd, 16, [1] * 7, [1, 2, 15, 16, 17, 100, 333], seed=heads)
    run("bf16", heads, kv_heads, hd, 8, [1, 0, 1], [9, 5, 64], seed=heads + 1, start=1, tail=2)
    run("bf16", heads, kv_heads, hd, 8, [1, 1], [0, 33], seed=heads + 2)


@pytest.mark.parametrize("io", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,hd,page", [(2, 2, 64, 16), (4, 1, 128, 64), (2, 1, 32, 8), (3, 3, 128, 8)])
def test_chunks(io, heads, kv_heads, hd, page):
    run(io, heads, kv_heads, hd, page, [1, 33, 64, 130, 0, 5, 2], [70, 33, 65, 200, 40, 3, 0], seed=hd, tail=1)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,length", [([128], [128]), ([127], [255]), ([129], [129]), ([256, 1], [513, 511]), ([300], [700]), ([1, 257], [1, 258])])
def test_chunk_borders(hd, new, length):
    run("bf16", 2, 2, hd, 32, new, length, seed=sum(new))


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_page_lengths(page, hd):
    run("bf16", 2, 2, hd, page, [1, 40], [page * 3 + 1, 150], seed=page)
    run("fp32", 2, 1, hd, page, [3], [page + 5], seed=page)


def test_long_sequences_are_split():
    run("fp32", 4, 2, 64, 64, [1, 1], [9001, 63], seed=5)
    run("bf16", 8, 1, 128, 128, [2], [7500], seed=6)
    run("bf16", 8, 1, 128, 128, [40], [6000], seed=7)
    run("bf16", 8, 1, 128, 16, [2], [7500], seed=6, max_len=0)        # the bound on lengths not given


@pytest.mark.parametrize("scale,k_gain,v_gain", [(0.05, 1.0, 1.0), (-0.3, 1.0, 1.0), (1.0, 4.0, 1.0), (None, 1e-6, 1e20), (1e-7, 1e6, 1e-20)])
@pytest.mark.parametrize("io", ["fp32", "bf16"])
def test_scales_and_magnitudes(scale, k_gain, v_gain, io):
    run(io, 2, 1, 64, 16, [1, 70], [50, 90], scale=scale, k_gain=k_gain, v_gain=v_gain, seed=11)


@pytest.mark.parametrize("io,out", [("fp32", "fp16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp16", "bf16")])
def test_output_types(io, out):
    run(io, 2, 2, 64, 16, [1, 70], [30, 100], out_dtype=out, seed=21)
    run(io, 2, 2, 128, 32, [1, 70], [30, 100], out_dtype=out, seed=22)


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_results_in_fp32_have_the_bits_of_two_fp16(io, hd):
    # one, some and many rows, split and not, on rows that begin at any element
    run(io, 2, 2, hd, 16, [1, 20, 70], [300, 200, 100], out_dtype="fp32", seed=31, fine=True)
    run(io, 4, 1, hd, 64, [130], [700], out_dtype="fp32", seed=32, fine=True)
    run(io, 2, 1, hd, 32, [49, 48, 47], [50, 333, 4000], out_dtype="fp32", seed=33, fine=True)


@pytest.mark.parametrize("new,length", [([1, 2], [100, 40]), ([90, 1], [100, 40])])
@pytest.mark.parametrize("hd", [64, 128])
def test_pages_that_do_not_exist_hide_their_keys(new, length, hd):
    lay = P.Layout(new, length, 16, seed=2)
    cache = P.make_cache(lay, 2, 2, hd, "e2m1")
    contents = F.fill(cache, lay, seed=3)
    gone = [(0, 1), (1, 0)]
    q = torch.randn(lay.n_tokens, 2, hd, generator=torch.Generator().manual_seed(4)).bfloat16()
    for s, i in gone:
        lay.pages[s, i] = -7 if s else lay.n_pages
    got = cache.attention(0, q.cuda(), lay.batch()).cpu().double()
    assert cache.status() == binding.STATUS_BAD_BATCH
    for r, s, p in lay.places():
        keep = torch.tensor([j for j in range(p + 1) if (s, j // 16) not in gone], dtype=torch.long)
        k, v = (x[:, keep] for x in contents[s])
        if not len(keep):
            assert bool((got[r] == 0).all())
            continue
        w = torch.softmax(torch.einsum("hd,hjd->hj", q[r].double(), k) * hd ** -0.5, -1)
        want = torch.einsum("hj,hjd->hd", w, v)
        # a bf16 result of bf16 weights: 2^-8 of the weights and of the scores' terms (below 40 in all), as in limit()
        assert float((got[r] - want).abs().max()) < 2.0 ** -8 * 3 * float(v.abs().max()), (r, s, p)


def test_queries_that_are_not_finite_stay_in_their_rows():
    lay = P.Layout([1, 66], [40, 66], 16, seed=2)
    cache = P.make_cache(lay, 2, 2, 64, "e2m1")
    F.fill(cache, lay, seed=3)
    q = torch.randn(lay.n_tokens, 2, 64, generator=torch.Generator().manual_seed(4)).bfloat16()
    clean = cache.attention(0, q.cuda(), lay.batch()).cpu().double()
    q[0, 1, 3] = float("nan")
    q[20, 0, 5] = float("nan")
    got = cache.attention(0, q.cuda(), lay.batch()).cpu().double()
    assert bool(torch.isnan(got[0, 1]).all()) and bool(torch.isnan(got[20, 0]).all())
    got[0, 1], got[20, 0] = clean[0, 1], clean[20, 0]
    assert not bool(torch.isnan(got).any())
    assert float((got - clean).abs().max()) < 2.0 ** -7 * float(clean.abs().max())


def test_captured_calls_follow_what_the_device_arrays_say():
    lay = P.Layout([1, 64, 1], [300, 120, 17], 16, seed=5, spare_columns=3)
    stream = torch.cuda.Stream()
    cache = P.make_cache(lay, 4, 4, 64, "e2m1", stream=stream)
    contents = F.fill(cache, lay, seed=6)
    g = torch.Generator().manual_seed(7)
    q = torch.randn(lay.n_tokens, 4, 64, generator=g).bfloat16().cuda()
    kv = torch.randn(2, lay.n_tokens, 4, 64, generator=g)
    batch = lay.batch(max_len=0)
    out = torch.zeros_like(q)
    rows = kv.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        cache.append(0, rows[0], rows[1], batch)
        cache.attention(0, q, batch, out=out)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cache.append(0, rows[0], rows[1], batch)
        cache.attention(0, q, batch, out=out)
    for seed in (8, 9):
        kv = torch.randn(2, lay.n_tokens, 4, 64, generator=torch.Generator().manual_seed(seed))
        rows.copy_(kv)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for r, s, p in lay.places():
            for i in (0, 1):
                contents[s][i][:, p] = F.stored(kv[i][r]).double()
        want, parts = P.attention(q.cpu(), contents, lay, 0.125, 1)
        got = out.cpu().double()
        assert bool(((got - want).abs() <= limit(want, parts, 64, torch.bfloat16)).all())
    assert cache.status() == 0


def test_the_same_call_gives_the_same_bits():
    lay = P.Layout([1, 1, 90], [9000, 500, 700], 64, seed=5)
    cache = P.make_cache(lay, 8, 2, 128, "e2m1")
    F.fill(cache, lay, seed=6)
    q = torch.randn(lay.n_tokens, 8, 128, generator=torch.Generator().manual_seed(7)).bfloat16().cuda()
    first = cache.attention(0, q, lay.batch())
    for _ in range(3):
        assert torch.equal(cache.attention(0, q, lay.batch()), first)
