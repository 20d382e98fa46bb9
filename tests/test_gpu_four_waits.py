"""Chunks over 4-bit pages whose kernel gives up a wait (the test hook): reported, nothing left behind, the next call as ever."""
import pytest
import torch

import four_reference as F
import paged_reference as P
import scores_reference as S
from paper_2307_02628_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 9.0])
def test_wait_that_expires_is_reported(io, hd, cap):
    lay = P.Layout([300], [600], 32, seed=1)
    cache = P.make_cache(lay, 2, 2, hd, "e2m1")
    contents = F.fill(cache, lay, seed=2)
    q = torch.randn(300, 2, hd, generator=torch.Generator().manual_seed(3)).to(P.TORCH[io])
    sc = binding.Scores(cap=cap) if cap else None
    cache.set_option(binding.SD_CACHE_OPT_TEST_WAIT_EXPIRY, 1)
    cache.attention(0, q.cuda(), lay.batch(), scores=sc)
    assert cache.status() & binding.STATUS_WAIT_EXPIRED
    got = cache.attention(0, q.cuda(), lay.batch(), scores=sc).cpu()
    assert cache.status() == 0
    want = S.reference(q, contents, lay, hd ** -0.5, 1, cap=cap)
    assert float(S.over(got, *want, hd, q.dtype, cap).max()) <= 1
