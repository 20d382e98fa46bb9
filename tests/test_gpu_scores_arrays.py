"""The rows' first and last visible positions at the end of a longer array: what lies behind them is another's."""
import pytest
import torch

import four_reference as F
import paged_reference as P
import scores_reference as S
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8", "e2m1"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
def test_masks_in_parts_of_longer_arrays(cache_dtype, hd, io):
    for n in (60, 128, 129, 300):                              # the last block: one tile of rows, or two
        lay = P.Layout([5, n], [40, n + 33], 16, seed=n)
        cache = P.make_cache(lay, 2, 2, hd, cache_dtype)
        contents = F.fill_any(cache, lay, seed=n + 1)
        g = torch.Generator().manual_seed(n + 2)
        q = torch.randn(lay.n_tokens, 2, hd, generator=g).to(P.TORCH[io])
        lo, hi = (torch.randint(0, n + 33, (lay.n_tokens,), generator=g) // d for d in (8, 1))
        around = torch.full((2, 300 + lay.n_tokens + 300), -(2 ** 31), dtype=torch.int32)
        outs = []
        for other in (-(2 ** 31), 2 ** 31 - 1):
            around[:] = other
            around[0, 300:-300], around[1, 300:-300] = lo, hi
            dev = around.cuda()
            outs.append(cache.attention(0, q.cuda(), lay.batch(), scores=binding.Scores(lo=dev[0, 300:-300], hi=dev[1, 300:-300])))
        assert cache.status() == 0
        assert torch.equal(*outs)
        want = S.reference(q, contents, lay, hd ** -0.5, 1, lo=lo, hi=hi)
        assert float(S.over(outs[0].cpu(), *want, hd, q.dtype).max()) <= 1
