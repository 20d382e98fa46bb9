"""Append to and read back from a paged cache in 4 bits: codes, block scales and scales equal to the 64-bit form's, values rounded once."""
import pytest
import torch

import four_reference as F
import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


def check_pools(cache, lay, k, v, layer=0):
    pool = {n: t.cpu() for n, t in cache.layer(layer).items()}
    for n, x in (("k", k), ("v", v)):
        code, block, scale = F.quantise(x.float())
        for r, s, p in lay.places():
            page, slot = lay.slot(s, p)
            have = F.values(F.unpack(pool[n][page, :, slot]), pool[n + "_block"][page, :, slot].view(torch.uint8), pool[n + "_scale"][page, :, slot])
            assert torch.equal(pool[n + "_scale"][page, :, slot], scale[r]), (n, r)
            assert torch.equal(pool[n + "_block"][page, :, slot].view(torch.uint8), block[r]), (n, r)
            assert torch.equal(have, F.values(code[r], block[r], scale[r])), (n, r)      # as values: -0 and 0 are one


def rows(lay, heads, hd, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(lay.n_tokens, heads, hd, generator=g) * torch.exp(torch.randn(lay.n_tokens, heads, hd // 16, generator=g)).repeat_interleave(16, -1)
    return (x * gain).to(P.TORCH[dtype])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kv_heads,hd,page", [(3, 64, 16), (1, 32, 8), (12, 128, 32), (5, 128, 8), (7, 32, 128), (2, 64, 64)])
def test_append_and_read_back(dtype, kv_heads, hd, page):
    lay = P.Layout([1, 0, 9, 33, 5], [17, 4, 9, 70, 3], page, seed=hd + page, start=1, tail=2)
    cache = P.make_cache(lay, kv_heads, kv_heads, hd, "e2m1", n_layers=2)
    k, v = rows(lay, kv_heads, hd, dtype, 1), rows(lay, kv_heads, hd, dtype, 2)
    for t in cache.layer(0).values():
        t.view(torch.uint8).fill_(0x33)
    cache.append(1, k.cuda(), v.cuda(), lay.batch())
    check_pools(cache, lay, k, v, layer=1)
    assert all(bool((t.view(torch.uint8) == 0x33).all()) for t in cache.layer(0).values())
    own = torch.zeros(lay.n_tokens, dtype=torch.bool)
    for s in range(len(lay.new)):
        own[int(lay.first[s]):int(lay.first[s + 1])] = True
    placed = {r for r, _, _ in lay.places()}
    for out_dtype in (torch.float32, torch.bfloat16, torch.float16):
        ko, vo = (torch.full(k.shape, 7.0, dtype=out_dtype, device="cuda") for _ in range(2))
        cache.read(1, lay.batch(), k=ko, v=vo)
        for got, x in ((ko, k), (vo, v)):
            want = torch.full(k.shape, 7.0, dtype=out_dtype)
            have = F.stored(x.float())
            for r in range(lay.n_tokens):
                if own[r]:
                    want[r] = have[r].clamp(-65504, 65504).to(out_dtype) if out_dtype == torch.float16 else have[r].to(out_dtype)
                    if r not in placed:
                        want[r] = 0
            assert torch.equal(got.cpu(), want), out_dtype
    assert cache.status() == 0
    cache.close()


def test_many_rows_share_blocks_of_the_kernel():
    lay = P.Layout([1400, 1211], [1500, 1211], 16, seed=4)           # enough rows for two per block
    cache = P.make_cache(lay, 2, 2, 64, "e2m1")
    k, v = rows(lay, 2, 64, "fp32", 1), rows(lay, 2, 64, "fp32", 2)
    cache.append(0, k.cuda(), v.cuda(), lay.batch())
    ko, vo = cache.read(0, lay.batch())
    assert torch.equal(ko.cpu(), F.stored(k)) and torch.equal(vo.cpu(), F.stored(v))


@pytest.mark.parametrize("how", ["slice", "heads first", "odd", "broadcast"])
def test_strided_rows(how):
    lay = P.Layout([5, 20], [9, 20], 8, seed=2)
    n, H, hd = lay.n_tokens, 3, 64
    cache = P.make_cache(lay, H, H, hd, "e2m1")
    g = torch.Generator().manual_seed(3)
    if how == "slice":
        wide = torch.randn(n, 3 * H * hd, generator=g).cuda()
        k, v = wide[:, H * hd:2 * H * hd].unflatten(1, (H, hd)), wide[:, 2 * H * hd:].unflatten(1, (H, hd))
    elif how == "heads first":
        k, v = (torch.randn(H, n, hd, generator=g).cuda().transpose(0, 1) for _ in range(2))
    elif how == "odd":
        k, v = (torch.randn(n, H, hd + 1, generator=g).bfloat16().cuda()[:, :, 1:] for _ in range(2))
    else:
        k, v = torch.randn(1, 1, hd, generator=g).cuda().expand(n, H, hd), torch.randn(n, 1, hd, generator=g).cuda().expand(n, H, hd)
    cache.append(0, k, v, lay.batch())
    check_pools(cache, lay, k.cpu(), v.cpu())
    big = torch.zeros(2, H, n, hd + 3, device="cuda")
    outs = [big[i, :, :, 1:hd + 1].transpose(0, 1) for i in range(2)]
    cache.read(0, lay.batch(), k=outs[0], v=outs[1])
    assert torch.equal(outs[0].cpu(), F.stored(k.cpu().float())) and torch.equal(outs[1].cpu(), F.stored(v.cpu().float()))


def test_borders_of_codes_and_of_block_scales():
    # rows whose scale is a power of two, elements on and next to the borders between codes; blocks next to borders between block scales
    hd, n = 128, 64
    lay = P.Layout([n], [n], 16, seed=1)
    mid = torch.cat([F.E2M1[1:], (F.E2M1[1:] + F.E2M1[:-1]) / 2]).float()                     # 14 numbers: codes and borders
    x = torch.zeros(n, 1, hd)
    for r in range(n):
        unit = 2.0 ** (r - 32)
        up, down = 1 + 2.0 ** -23, 1 - 2.0 ** -24
        for b in range(8):
            part = torch.zeros(16)
            part[0] = 6.0 * [1.0, up, down, 1.0, up, down, 1.0, 1.0][b] * float(F.E4M3[126 - 9 * b])      # the block's largest
            part[1:15] = mid[torch.randperm(14, generator=torch.Generator().manual_seed(r * 8 + b))] * float(F.E4M3[126 - 9 * b]) * [1.0, up, down][(r + b) % 3]
            part[2::2] *= -1
            x[r, 0, 16 * b:16 * b + 16] = part * unit
        if r % 2:                                                # and block scales between two of them
            x[r, 0, 16:32] = 0
            x[r, 0, 17] = 6.0 * float((F.E4M3[100] + F.E4M3[101]) / 2) * unit * [1.0, up, down][r % 3]
    cache = P.make_cache(lay, 1, 1, hd, "e2m1")
    cache.append(0, x.cuda(), -x.cuda(), lay.batch())
    check_pools(cache, lay, x, -x)
    assert cache.status() == 0


def test_extreme_rows():
    hd = 64
    lay = P.Layout([10], [10], 16, seed=1)
    g = torch.Generator().manual_seed(8)
    x = torch.randn(10, 1, hd, generator=g)
    x[0] = 0
    x[1] *= 1e-42                                                # scales that are subnormal, or 0 although elements are not
    x[2] *= 1e-38
    x[3] = 3.4e38 * torch.sign(x[3])
    x[4] *= 1e-30
    x[5, 0, 16:] *= 1e-9                                         # blocks far below the row's largest: their scale rounds to 0
    x[6, 0, :16] = 0
    x[7, 0, 5:] = 0
    x[8] *= 1e30
    x[9, 0, 16:32] *= 2.0 ** -16
    cache = P.make_cache(lay, 1, 1, hd, "e2m1")
    cache.append(0, x.cuda(), x.cuda(), lay.batch())
    check_pools(cache, lay, x, x)
    assert cache.status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_elements_that_are_not_finite(dtype):
    hd = 32
    lay = P.Layout([6], [6], 8, seed=1)
    g = torch.Generator().manual_seed(9)
    x = torch.randn(6, 1, hd, generator=g)
    x[0, 0, 3] = float("inf")
    x[1, 0, 20] = float("-inf")
    x[2, 0, 7] = float("nan")
    x[3] = float("nan")
    x[4] = float("inf")
    x[5, 0, ::2] = float("nan")
    x[5, 0, 1] = float("inf")
    x = x.to(P.TORCH[dtype])
    cache = P.make_cache(lay, 1, 1, hd, "e2m1")
    cache.append(0, x.cuda(), torch.zeros_like(x).cuda(), lay.batch())
    check_pools(cache, lay, x, torch.zeros_like(x))
    assert cache.status() == binding.STATUS_NOT_FINITE
    ko, _ = cache.read(0, lay.batch())
    assert bool(torch.isfinite(ko).all())
    assert float(ko[0, 0, 3]) == float(ko[0].abs().max())


def test_bad_pages_and_places_are_skipped():
    lay = P.Layout([4, 3], [20, 9], 8, seed=3)
    lay.pages[0, 2] = lay.n_pages + 5
    lay.pages[1, 0] = -3
    cache = P.make_cache(lay, 2, 2, 64, "e2m1")
    for t in cache.layer(0).values():
        t.view(torch.uint8).fill_(0x22)
    x = rows(lay, 2, 64, "fp32", 1)
    cache.append(0, x.cuda(), x.cuda(), lay.batch())
    assert cache.status() == binding.STATUS_BAD_BATCH
    k, _ = cache.read(0, lay.batch())
    assert cache.status() == binding.STATUS_BAD_BATCH
    assert bool((k[:6] == 0).all())                                  # positions 16..19 of the first, 6 and 7 of the second
    assert torch.equal(k[6].cpu(), F.stored(x)[6])
