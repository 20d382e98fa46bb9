"""Results in fp32 over many keys: sums that do not shrink.

Queries are zeros and all values one number, so that every weight is 1 and their sum a whole number: what a result is off by is its sum over the values.  A
tensor core's addition of 16 products truncates each of them, and the sum so far, to a multiple of the last place: 2^-23 of the sum at most.  The kernel for chunks makes a
sum of 256 keys of 16 additions of the weights' first parts and as many of their second ones.  A first part (11 bits) times 2688 (21 * 2^7) has 16 bits, of a sum of at most 256
such products all 24: nothing is lost but by the sum so far, 32 times.  Of a second part's products each may lose as much: 16 * 16.  Half of it all, as the sum grows evenly.
Then sums of 256 keys are added, rounded to nearest: half of n / 256 * 2^-24; the weight's second part is rounded to 2^-23, and two more products to 2^-24 each.
"""
import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,new,length", [(4, 64, 4096), (32, 64, 16384), (1, 300, 30000), (2, 130, 1000)])
@pytest.mark.parametrize("value", [1.0, -0.7, 1.9])
@pytest.mark.parametrize("masked", [False, True])
def test_sums_over_many_keys(hd, heads, new, length, value, masked):
    lay = P.Layout([new], [length], 64, seed=1)
    cache = P.make_cache(lay, heads, heads, hd, "e2m1")
    pool = cache.layer(0)
    for n, t in pool.items():                                  # keys of zeros; every value the largest code, block scale and a scale to make it `value`
        t.view(torch.uint8).zero_() if n[0] == "k" else t.copy_(torch.tensor(value).abs() / 2688) if n == "v_scale" else t.view(torch.uint8).fill_(
            0x7e if n == "v_block" else 0x77 if value > 0 else 0xff)
    scale = float(pool["v_scale"].flatten()[0])
    lo = torch.full((new,), 70, dtype=torch.int32).cuda() if masked else None
    sc = binding.Scores(lo=lo) if masked else None
    out = cache.attention(0, torch.zeros(new, heads, hd, device="cuda"), lay.batch(), scores=sc).cpu().double()
    assert cache.status() == 0
    want = 2688 * scale * (1 if value > 0 else -1)
    limit = (16 * 16 + 32) / 2 * 2.0 ** -23 + length / 512 * 2.0 ** -24 + 2.0 ** -22
    assert float((out / want - 1).abs().max()) <= limit, (float((out / want - 1).abs().max()), limit)
