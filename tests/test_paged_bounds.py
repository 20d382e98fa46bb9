"""The limits of the attention tests tell right from wrong: an emulation of the kernels' roundings stays inside, the mistakes that split
keys, masks, pages and joins can make do not."""
import pytest
import torch

import paged_bounds as B
import paged_reference as P


def emulate(q, contents, layout, scale, group, seen_of, twice=None):
    """Attention with the weights of each row rounded to bf16 (relative to the row's maximum) and the result rounded to q's type; seen_of(s,
    position, length): the keys that a row sums over; twice: keys that enter a second time."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    for r, s, p in layout.places():
        k, v = contents[s]
        x = torch.einsum("kgd,kjd->kgj", q[r].double().view(k.shape[0], group, -1), k) * scale
        x = x.masked_fill(~seen_of(s, p, k.shape[1]), float("-inf"))
        w = torch.exp(x - x.amax(-1, keepdim=True))
        if twice is not None:
            w = w * (1.0 + twice(k.shape[1]).double())
        rounded = w.bfloat16().double() if q.dtype == torch.bfloat16 else w
        out[r] = (torch.einsum("kgj,kjd->kgd", rounded, v) / w.sum(-1, keepdim=True)).reshape(out[r].shape)
    return out.to(q.dtype)


CASES = [([20, 9], [2900, 700], 4, 1, 64), ([13], [3333], 7, 1, 128), ([24, 3], [900, 129], 2, 2, 64)]


@pytest.mark.parametrize("new,length,heads,kv_heads,hd", CASES)
@pytest.mark.parametrize("io", ["bf16", "fp16"])
def test_the_limit_sees_one_key(new, length, heads, kv_heads, hd, io):
    lay = P.Layout(new, length, 32, seed=1)
    contents = B.contents_of(lay, kv_heads, hd, 2)
    q = torch.randn(lay.n_tokens, heads, hd, generator=torch.Generator().manual_seed(3)).to(P.TORCH[io])
    scale, group = hd ** -0.5, heads // kv_heads
    ref = B.reference(q, contents, lay, scale, group)
    keys = lambda n: torch.arange(n)  # noqa: E731

    def worst(seen, **kw):
        o = B.over(emulate(q, contents, lay, scale, group, seen, **kw), *ref, hd, q.dtype)
        return float(o.max()), float(o.median())

    right = lambda s, p, n: keys(n) <= p  # noqa: E731
    assert worst(right)[0] < 1
    assert float(B.over(torch.zeros_like(q), *ref, hd, q.dtype).min()) > 10
    # what a lost tile, split, page or half of a tile leaves out, in any row
    assert worst(lambda s, p, n: (keys(n) <= p) & ~((keys(n) >= 64) & (keys(n) < 128)))[1] > 1
    assert worst(right, twice=lambda n: (keys(n) >= 64) & (keys(n) < 128))[1] > 1
    # one key: the row's own, the next one, the last of a tile, the first of one
    for missing in (lambda n, p: keys(n) == p, lambda n, p: keys(n) == 63, lambda n, p: keys(n) == 64):
        assert worst(lambda s, p, n, m=missing: (keys(n) <= p) & ~m(n, p))[0] > 1
    assert worst(lambda s, p, n: keys(n) <= p + 1)[0] > 1
