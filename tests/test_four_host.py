"""CPU-only checks of the 4-bit cache: sizes, refusals, and the plain form that the GPU tests compare with."""
import ctypes as C

import pytest
import torch

import four_reference as F
from paper_2307_02628_b200 import binding


def config(**kw):
    base = dict(n_layers=2, n_heads=8, n_kv_heads=4, head_dim=64, page_len=16, n_pages=10, max_seqs=3, max_tokens=50, dtype=binding.SD_DTYPE_E2M1)
    return binding.SdCacheConfig(*[{**base, **kw}[n] for n, _ in binding.SdCacheConfig._fields_])


@pytest.mark.parametrize("n_pages", [10, 10 ** 6])
@pytest.mark.parametrize("head_dim", [32, 64, 128])
def test_the_arena_holds_the_pools(n_pages, head_dim):
    pools = 2 * 2 * n_pages * 4 * 16 * (head_dim // 2 + head_dim // 16 + 4)
    assert pools <= binding.cache_bytes(config(n_pages=n_pages, head_dim=head_dim)) <= pools + (1 << 26)


@pytest.mark.parametrize("bad", [dict(head_dim=16), dict(head_dim=48), dict(page_len=4), dict(n_pages=0), dict(dtype=7), dict(dtype=5)])
def test_configurations_that_are_refused(bad):
    with pytest.raises(binding.SdError) as e:
        binding.cache_bytes(config(**bad))
    assert e.value.code == binding.SD_ERR_ARG


def test_no_cache_no_blocks():
    L = binding.lib()
    p = C.c_void_p()
    assert L.sd_cache_layer_blocks(None, 0, C.byref(p), None) == binding.SD_ERR_ARG


def test_plain_form_by_exhaustive_search():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 64, generator=g) * torch.exp(2 * torch.randn(40, 1, generator=g))
    code, block, scale = F.quantise(x)
    top = x.double().abs().unflatten(-1, (-1, 16)).amax(-1)
    want = (F.E4M3.view(1, 1, -1) * 6 * scale.double().view(-1, 1, 1) - top.unsqueeze(-1)).abs().min(-1).values
    got = (F.E4M3[block.long()] * 6 * scale.double().unsqueeze(-1) - top).abs()
    assert torch.allclose(got, want, rtol=1e-12, atol=0)
    signed = torch.cat([F.E2M1, -F.E2M1])
    unit = (F.E4M3[block.long()] * scale.double().unsqueeze(-1)).repeat_interleave(16, -1)
    want = (signed.view(1, 1, -1) * unit.unsqueeze(-1) - x.double().unsqueeze(-1)).abs().min(-1).values
    assert torch.allclose((F.values(code, block, scale) - x.double()).abs(), want, rtol=1e-12, atol=1e-300)
    assert torch.equal(F.unpack(F.pack(code)), code)
    # the row's largest element comes back as scale * 2688: its block has the largest block scale and its code is 6
    assert torch.equal(F.values(code, block, scale).abs().amax(-1), 2688 * scale.double())


def test_ties_go_to_the_even_code():
    y = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], dtype=torch.float64)
    assert F.E2M1[F.nearest(y, F.E2M1)].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    assert float(F.E4M3[-1]) == 448.0 and len(F.E4M3) == 127
