"""A bias by distance is slope times a whole number, rounded once: seen through weights that come out one by one.

Queries are zeros, and the value of position j is a one at element j mod 64: with a window of 64, element j mod 64 of a result is the weight of position j.
Two weights of a row differ by e^(-slope distance); the sum that both are divided by drops out of their quotient.
Its relative error, over a cache in 4 bits with results in fp32: for either weight 2^-22 of the exponential, 2^-22 of a pair of fp16, 2^-23 of its product with
the value's scale and of the result; in an exponent of b (in base 2) 2^-24 b of slope log2 e, as much of log2 e itself, of the bias, half of it of a sum, and
2^-24 (b + 8) of the difference to the running maximum, which may be 8 behind.
"""
import math

import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ahead", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_weights_of_one_row(ahead, page):
    slopes = torch.tensor([4.0, 2.0, 1.0, 0.25, 0.7, 0.03])
    heads, n, length = len(slopes), 400, 1000
    lay = P.Layout([n], [length], page, seed=1)
    cache = P.make_cache(lay, heads, heads, 64, "e2m1")
    everything = P.Layout([length], [length], page, seed=1)
    store = P.make_cache(everything, heads, heads, 64, "e2m1")     # of the same shape, for more rows a call
    ones = torch.eye(64)[torch.arange(length) % 64].unsqueeze(1).expand(length, heads, 64).contiguous().cuda()
    store.append(0, torch.randn(length, heads, 64).cuda(), ones, everything.batch())
    for name, t in store.layer(0).items():
        cache.layer(0)[name].view(torch.uint8).copy_(t.view(torch.uint8))
    hi = torch.full((n,), length - 1, dtype=torch.int32).cuda() if ahead else None
    sc = binding.Scores(slopes=slopes.cuda(), window=64, hi=hi)
    out = cache.attention(0, torch.zeros(n, heads, 64, device="cuda"), lay.batch(), scores=sc).cpu().double()
    assert cache.status() == 0 and store.status() == 0
    p = torch.arange(length - n, length)
    if ahead:                                                      # only rows whose elements are of one position each
        rows = torch.tensor([n - 1])
    else:
        rows = torch.arange(n)
    own = out[rows, :, p[rows] % 64]
    worst = 0.0
    for d in range(1, 64):
        b = slopes.double() * d / math.log(2)
        limit = 2 * (2.0 ** -22 + 2.0 ** -22 + 2.0 ** -23) + math.log(2) * 2.0 ** -24 * (4.5 * b + 8)
        got = out[rows, :, (p[rows] - d) % 64] / own
        over = (got / torch.exp(-slopes.double() * d) - 1).abs().amax(0) / limit
        worst = max(worst, float((over * (slopes * d <= 5)).max()))       # weights that fp16 holds as normal numbers
    assert worst <= 1, worst
