"""Storing keys and values in a paged cache and reading them back, against the 64-bit form, bit for bit."""
import ctypes as C

import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu

CACHES = ("fp32", "bf16", "int8", "e4m3")


def _rows(layout, heads, hd, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(layout.n_tokens, heads, hd, generator=g) * gain).to(dtype)


def _check_pools(cache, layout, k, v, layer=0, before=None):
    """Every place holds what the definition says; every other place is as it was."""
    dtype = {0: "fp32", 1: "bf16", 3: "int8", 4: "e4m3"}[cache.cfg.dtype]
    pool = {n: t.cpu() for n, t in cache.layer(layer).items()}
    want = {n: t.clone() for n, t in before.items()}
    for n, x in (("k", k), ("v", v)):
        if dtype in P.TOP:
            codes, scale = P.quantise(x.float(), dtype)
            codes = codes.to(P.TORCH[dtype])
        else:
            codes = P.stored(x, dtype).to(P.TORCH[dtype])
        for r, s, p in layout.places():
            page, slot = layout.slot(s, p)
            want[n][page, :, slot] = codes[r]
            if dtype in P.TOP:
                want[n + "_scale"][page, :, slot] = scale[r]
    for n in pool:
        if pool[n].dtype == torch.float8_e4m3fn:                 # -0 and 0 are one value, compared as values
            assert torch.equal(pool[n].float().nan_to_num(9e9), want[n].float().nan_to_num(9e9)), n
        else:
            assert torch.equal(pool[n].float().nan_to_num(9e9), want[n].float().nan_to_num(9e9)), n


def _poison(cache, layer=0):
    """All bits set: NaN in every float type, so that whatever is written by mistake shows."""
    for t in cache.layer(layer).values():
        t.view(torch.uint8).fill_(255)
    return {n: t.cpu().clone() for n, t in cache.layer(layer).items()}


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("rows_dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kv_heads,hd,page", [(1, 32, 8), (3, 64, 16), (5, 128, 32), (32, 128, 128)])
def test_append_and_read_back(cache_dtype, rows_dtype, kv_heads, hd, page):
    lay = P.Layout([1, 0, 7, 40, 1], [1, 3, 7, 90, 2 * page], page, seed=hd, start=2, tail=3)
    cache = P.make_cache(lay, kv_heads, kv_heads, hd, cache_dtype, n_layers=2)
    before = _poison(cache, 1)
    k, v = (_rows(lay, kv_heads, hd, P.TORCH[rows_dtype], seed, 3.0) for seed in (1, 2))
    b = lay.batch()
    cache.append(1, k.cuda(), v.cuda(), b)
    torch.cuda.synchronize()
    _check_pools(cache, lay, k, v, 1, before)
    for out_dtype in (torch.float32, torch.bfloat16, torch.float16):
        ko = torch.full(k.shape, 77.0, dtype=out_dtype, device="cuda")
        vo = torch.full(k.shape, 78.0, dtype=out_dtype, device="cuda")
        cache.read(1, b, k=ko, v=vo)
        for x, got, mark in ((k, ko, 77.0), (v, vo, 78.0)):
            want = torch.full(k.shape, mark, dtype=out_dtype)
            have = P.stored(x.float(), cache_dtype)
            for r, _, _ in lay.places():
                want[r] = have[r].clamp(-65504, 65504).to(out_dtype) if out_dtype == torch.float16 else have[r].to(out_dtype)
            assert torch.equal(got.cpu(), want)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("how", ["qkv", "odd", "head-major", "broadcast"])
def test_append_from_strided_rows_and_read_into_them(cache_dtype, how):
    lay = P.Layout([5, 1, 9], [6, 1, 20], 16, seed=4)
    H, hd, n = 4, 64, 15
    cache = P.make_cache(lay, H, H, hd, cache_dtype)
    before = _poison(cache)
    g = torch.Generator().manual_seed(3)
    if how == "qkv":                                            # slices of wider rows
        wide = torch.randn(n, 3 * H * hd, generator=g).bfloat16()
        cut = lambda t: (t[:, H * hd:2 * H * hd].unflatten(1, (H, hd)), t[:, 2 * H * hd:].unflatten(1, (H, hd)))  # noqa: E731
    elif how == "odd":                                          # nothing is 16-byte aligned
        wide = torch.randn(2, n, H, hd + 1, generator=g)
        cut = lambda t: (t[0][..., 1:], t[1][..., 1:])  # noqa: E731
    elif how == "head-major":
        wide = torch.randn(2, H, n, hd, generator=g).half()
        cut = lambda t: (t[0].transpose(0, 1), t[1].transpose(0, 1))  # noqa: E731
    else:                                                       # one head for all
        wide = torch.randn(2, n, 1, hd, generator=g)
        cut = lambda t: (t[0].expand(n, H, hd), t[1].expand(n, H, hd))  # noqa: E731
    k, v = cut(wide.cuda())
    cache.append(0, k, v, lay.batch())
    torch.cuda.synchronize()
    kc, vc = cut(wide)
    _check_pools(cache, lay, kc, vc, 0, before)
    if how != "broadcast":
        into = torch.zeros_like(wide, device="cuda")
        ko, vo = cut(into)
        cache.read(0, lay.batch(), k=ko, v=vo)
        want = torch.zeros_like(wide)
        cut(want)[0].copy_(P.stored(kc.float(), cache_dtype))
        cut(want)[1].copy_(P.stored(vc.float(), cache_dtype))
        assert torch.equal(into.cpu(), want)
    else:
        with pytest.raises(binding.SdError):                    # an output's heads may not overlap
            cache.read(0, lay.batch(), k=k, v=v)
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["int8", "e4m3"])
def test_codes_at_borders_and_extreme_rows(cache_dtype):
    # every border between two codes, and the floats next to it, for scales that are powers of two and others
    top = P.TOP[cache_dtype]
    if cache_dtype == "int8":
        borders = torch.arange(-127, 127).float() + 0.5
    else:
        v = torch.arange(0, 0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
        borders = torch.cat([(v[1:] + v[:-1]) / 2, -(v[1:] + v[:-1]) / 2])
    rows = []
    for scale in (1.0, 0.25, 3.0, 0.1, 1.7e-3, 2.0 ** -100, 1e30, 1.3e-38, 3e-42):
        s = torch.tensor(top, dtype=torch.float32) * scale / top
        x = borders.double() * float(s)
        x = x.float()
        x = torch.cat([x, torch.nextafter(x, torch.tensor(float("inf"))), torch.nextafter(x, torch.tensor(-float("inf")))])
        x = x[x.abs() <= top * s]
        x = torch.cat([x, torch.zeros((-len(x)) % 127)]).view(-1, 127)
        rows.append(torch.cat([torch.full((len(x), 1), float(top * s)), x], 1))
    rows = torch.cat(rows)
    rows = torch.cat([rows, torch.zeros(1, 128), torch.full((1, 128), 1e-45), torch.full((1, 128), -3.4e38)])
    odd = torch.randn(4, 128)
    odd[0, 3], odd[1, 4], odd[2, 5] = float("inf"), float("-inf"), float("nan")
    odd[3] = float("nan")
    for x, status in ((rows, 0), (odd, binding.STATUS_NOT_FINITE)):
        n = len(x)
        lay = P.Layout([n], [n], 16)
        cache = P.make_cache(lay, 1, 1, 128, cache_dtype)
        before = _poison(cache)
        k, v = x.unsqueeze(1), x.flip(0).unsqueeze(1)
        cache.append(0, k.cuda(), v.cuda().contiguous(), lay.batch())
        torch.cuda.synchronize()
        _check_pools(cache, lay, k, v, 0, before)
        assert cache.status() == status
        assert cache.status() == 0                              # read and cleared
        cache.close()


@pytest.mark.parametrize("cache_dtype", ["fp32", "bf16"])
def test_values_that_are_not_finite_are_stored_as_finite_ones(cache_dtype):
    lay = P.Layout([2], [2], 8)
    cache = P.make_cache(lay, 1, 1, 32, cache_dtype)
    before = _poison(cache)
    x = torch.randn(2, 1, 32)
    x[0, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.4028234e38])
    cache.append(0, x.cuda(), x.cuda(), lay.batch())
    torch.cuda.synchronize()
    _check_pools(cache, lay, x, x, 0, before)
    assert cache.status() == binding.STATUS_NOT_FINITE
    cache.close()


def test_what_the_device_finds_wrong_is_reported_and_skipped():
    H, hd = 2, 64
    lay = P.Layout([3, 4, 2], [3, 20, 30], 16, tail=1)
    cache = P.make_cache(lay, H, H, hd, "int8")
    k, v = _rows(lay, H, hd, torch.float32, 1).cuda(), _rows(lay, H, hd, torch.float32, 2).cuda()

    def run(change):
        before = _poison(cache)
        pages, first, length = lay.pages.clone(), lay.first.clone(), lay.len.clone()
        max_new = change(pages, first, length) or 4
        b = binding.CacheBatch(pages.cuda(), first.cuda(), length.cuda(), lay.n_tokens, max_new)
        cache.append(0, k, v, b)
        out = cache.read(0, b, k=torch.full(k.shape, 5.0, device="cuda"), v=torch.full(k.shape, 5.0, device="cuda"))[0].cpu()
        pool = cache.layer(0)["k_scale"].cpu()
        written = int((~torch.isnan(pool[:, 0])).sum())
        assert int((~torch.isnan(before["k_scale"])).sum()) == 0
        return cache.status(), written, out

    status, written, out = run(lambda p, f, l: None)
    assert status == 0 and written == 9 and bool((out[9] == 5).all())

    def bad_page(p, f, l):
        p[1, 1] = lay.n_pages                                    # one past the pool: positions 16..19 of sequence 1
    status, written, out = run(bad_page)
    assert status == binding.STATUS_BAD_BATCH and written == 5 and bool((out[3:7] == 0).all())

    def negative_page(p, f, l):
        p[0, 0] = -7
    status, written, out = run(negative_page)
    assert status == binding.STATUS_BAD_BATCH and written == 6 and bool((out[:3] == 0).all())

    def too_long(p, f, l):
        l[2] = lay.columns * 16 + 1                              # the last token lies past the table
    status, written, out = run(too_long)
    assert status & binding.STATUS_BAD_BATCH and bool((out[8] == 0).all())

    def beyond_rows(p, f, l):
        f[3] = lay.n_tokens + 5
        l[2] = 30
    status, written, out = run(beyond_rows)
    assert status == binding.STATUS_BAD_BATCH

    def falling(p, f, l):
        f[1], f[2] = 7, 3                                        # not in order
    assert run(falling)[0] == binding.STATUS_BAD_BATCH

    def short_bound(p, f, l):
        return 2                                                 # max_new below what sequences 0 and 1 bring
    status, written, out = run(short_bound)
    assert status == binding.STATUS_BAD_BATCH and written == 6 and bool((out[2] == 5).all())

    def shorter_than_new(p, f, l):
        l[1] = 2                                                 # two of the four new tokens have no place: no error
    status, written, out = run(shorter_than_new)
    assert status == 0 and written == 7 and bool((out[3:5] == 0).all())

    def empty(p, f, l):
        l[1] = 0
    status, written, out = run(empty)
    assert status == 0 and written == 5 and bool((out[3:7] == 0).all())
    cache.close()


def test_refusals():
    lay = P.Layout([2, 1], [2, 9], 16)
    cache = P.make_cache(lay, 4, 2, 64, "int8")
    k = torch.zeros(3, 2, 64, device="cuda")
    q = torch.zeros(3, 4, 64, device="cuda")
    b = lay.batch()
    for call in (lambda: cache.append(1, k, k, b), lambda: cache.append(-1, k, k, b), lambda: cache.read(1, b),
                 lambda: cache.attention(1, q, b), lambda: cache.layer(1), lambda: cache.append(0, k, k.half(), b)):
        with pytest.raises(binding.SdError) as e:
            call()
        assert e.value.code == binding.SD_ERR_ARG
    for call in (lambda: cache.append(0, k.cpu(), k, b), lambda: cache.append(0, k.double(), k, b), lambda: cache.append(0, k[:2], k, b),
                 lambda: cache.attention(0, k, b), lambda: cache.append(0, k.transpose(1, 2).contiguous().transpose(1, 2), k, b),
                 lambda: cache.attention(0, q, b, scale=float("nan")), lambda: cache.attention(0, q, b, scale=0.0)):
        with pytest.raises(ValueError):
            call()
    L = binding.lib()
    rows = binding.SdHeads(k.data_ptr(), k.stride(0), k.stride(1), binding.SD_DTYPE_FP32)
    for field, value, code in (("pages", None, binding.SD_ERR_ARG), ("first", None, binding.SD_ERR_ARG), ("len", None, binding.SD_ERR_ARG),
                               ("n_seqs", 0, binding.SD_ERR_ARG), ("n_seqs", 9, binding.SD_ERR_CAPACITY), ("pages_per_seq", 0, binding.SD_ERR_ARG),
                               ("pages_per_seq", 1 << 30, binding.SD_ERR_ARG), ("n_tokens", -1, binding.SD_ERR_ARG), ("n_tokens", 9, binding.SD_ERR_CAPACITY),
                               ("max_new", 0, binding.SD_ERR_ARG), ("max_new", 4, binding.SD_ERR_ARG), ("max_len", -1, binding.SD_ERR_ARG)):
        c = binding.SdBatch.from_buffer_copy(b.c)
        setattr(c, field, value)
        assert L.sd_cache_append(cache.h, 0, C.byref(c), C.byref(rows), C.byref(rows)) == code, field
    for field, value in (("data", None), ("data", rows.data + 1), ("row_stride", -1), ("head_stride", -1), ("dtype", binding.SD_DTYPE_INT8),
                         ("row_stride", 1 << 60)):
        bad = binding.SdHeads.from_buffer_copy(rows)
        setattr(bad, field, value)
        assert L.sd_cache_append(cache.h, 0, C.byref(b.c), C.byref(bad), C.byref(rows)) == binding.SD_ERR_ARG, field
        assert L.sd_cache_append(cache.h, 0, C.byref(b.c), C.byref(rows), C.byref(bad)) == binding.SD_ERR_ARG, field
    # nothing to do is no error
    none = binding.CacheBatch(lay.pages.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), lay.len.cuda(), 0, 0)
    cache.append(0, k[:0], k[:0], none)
    assert cache.attention(0, q[:0], none).shape == (0, 4, 64)
    assert cache.status() == 0
    cache.close()


@pytest.mark.parametrize("cache_dtype", ["fp32", "int8"])
def test_tables_reach_at_most_two_to_the_thirtieth_positions(cache_dtype):
    # key numbers are 32-bit in the kernels; the table's entries past the sequence's end are not read, so none have to be there
    lay = P.Layout([2], [9], 16)
    cache = P.make_cache(lay, 2, 2, 64, cache_dtype)
    x = torch.ones(2, 2, 64, device="cuda")
    L = binding.lib()
    rows = binding.SdHeads(x.data_ptr(), x.stride(0), x.stride(1), binding.SD_DTYPE_FP32)
    b = lay.batch()
    cache.append(0, x, x, b)
    for columns, code in (((1 << 30) // 16, binding.SD_OK), ((1 << 30) // 16 + 1, binding.SD_ERR_ARG), ((1 << 31) // 16 - 1, binding.SD_ERR_ARG)):
        c = binding.SdBatch.from_buffer_copy(b.c)
        c.pages_per_seq = columns
        for call in (lambda: L.sd_cache_append(cache.h, 0, C.byref(c), C.byref(rows), C.byref(rows)),
                     lambda: L.sd_cache_read(cache.h, 0, C.byref(c), C.byref(rows), C.byref(rows)),
                     lambda: L.sd_cache_attention(cache.h, 0, C.byref(c), C.byref(rows), 0.0, C.byref(rows))):
            assert call() == code
    torch.cuda.synchronize()
    # the length hint may be anything: it only guides how the work is split
    pool = P.fill(cache, lay, seed=3)
    q = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(4))
    want, parts = P.attention(q, pool, lay, 0.125, 1)
    lim = P.bound(want, parts, 2.0 ** -15, 2.0 ** -15, torch.float32)      # operands of 16 bits (2^-16), the sums' roundings below that
    for hint in (0, 9, 2 ** 31 - 1):
        got = cache.attention(0, q.cuda(), lay.batch(max_len=hint)).cpu().double()
        assert bool(((got - want).abs() <= lim).all())
    assert cache.status() == 0
    cache.close()


def test_scales_that_fp32_does_not_hold_are_refused():
    # one that is 0 in fp32 would stand for the default
    lay = P.Layout([2], [9], 16)
    cache = P.make_cache(lay, 2, 2, 64, "bf16")
    P.fill(cache, lay, seed=1)
    q = torch.ones(2, 2, 64, device="cuda")
    for scale in (1e-60, -1e-46, 1e39, float("inf"), 0.0, float("nan")):
        with pytest.raises(ValueError):
            cache.attention(0, q, lay.batch(), scale=scale)
    with pytest.raises(binding.SdError) as e:
        cache.attention(0, q, lay.batch(), scale=3e38)          # infinite once it is turned to base 2
    assert e.value.code == binding.SD_ERR_ARG
    tiny = cache.attention(0, q, lay.batch(), scale=1e-40)      # all keys alike
    assert not torch.equal(tiny, cache.attention(0, q, lay.batch()))
    assert cache.status() == 0
    cache.close()
