"""CPU-only checks of the paged cache: sizes, refusals, the index arithmetic of the batch description, the plain forms the GPU tests use."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding, build


def config(**kw):
    base = dict(n_layers=2, n_heads=8, n_kv_heads=4, head_dim=64, page_len=16, n_pages=10, max_seqs=3, max_tokens=50, dtype=binding.SD_DTYPE_INT8)
    return binding.SdCacheConfig(*[{**base, **kw}[n] for n, _ in binding.SdCacheConfig._fields_])


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(n_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(head_dim=48), dict(head_dim=256),
                                 dict(page_len=4), dict(page_len=24), dict(page_len=256), dict(n_pages=0), dict(n_pages=-1), dict(max_seqs=0),
                                 dict(max_tokens=0), dict(dtype=binding.SD_DTYPE_FP16), dict(dtype=5), dict(dtype=-1), dict(n_heads=65536),
                                 dict(n_layers=2 ** 31 - 1, n_pages=2 ** 31 - 1, page_len=128)])
def test_configurations_that_are_refused(bad):
    with pytest.raises(binding.SdError) as e:
        binding.cache_bytes(config(**bad))
    assert e.value.code == binding.SD_ERR_ARG


@pytest.mark.parametrize("dtype,element,scales", [(binding.SD_DTYPE_FP32, 4, 0), (binding.SD_DTYPE_BF16, 2, 0), (binding.SD_DTYPE_INT8, 1, 4),
                                                   (binding.SD_DTYPE_E4M3, 1, 4)])
def test_the_arena_holds_the_pools(dtype, element, scales):
    for n_pages in (10, 10 ** 6):                               # the second: pools beyond 2^32 bytes
        pools = 2 * 2 * n_pages * 4 * 16 * (64 * element + scales)
        assert pools <= binding.cache_bytes(config(dtype=dtype, n_pages=n_pages)) <= pools + (1 << 26)


def test_null_arguments_are_refused():
    L = binding.lib()
    n = C.c_size_t()
    out = C.c_void_p()
    cfg = config()
    assert L.sd_cache_bytes(None, C.byref(n)) == binding.SD_ERR_ARG
    assert L.sd_cache_bytes(C.byref(cfg), None) == binding.SD_ERR_ARG
    assert L.sd_cache_create(C.byref(cfg), None, 1 << 30, None, C.byref(out)) == binding.SD_ERR_ARG
    assert L.sd_cache_create(C.byref(cfg), 4096 + 8, 1 << 30, None, C.byref(out)) == binding.SD_ERR_ARG      # not 256-byte aligned
    assert L.sd_cache_create(C.byref(cfg), 4096, 100, None, C.byref(out)) == binding.SD_ERR_CAPACITY
    b, r = binding.SdBatch(), binding.SdHeads()
    for call in (lambda: L.sd_cache_append(None, 0, C.byref(b), C.byref(r), C.byref(r)), lambda: L.sd_cache_read(None, 0, C.byref(b), C.byref(r), C.byref(r)),
                 lambda: L.sd_cache_attention(None, 0, C.byref(b), C.byref(r), 0.0, C.byref(r)), lambda: L.sd_cache_layer(None, 0, None, None, None, None),
                 lambda: L.sd_cache_status(None, None), lambda: L.sd_extend(None, None, None, None, 1, 0, None),
                 lambda: L.sd_sample(None, None, 1, None, None, None)):
        assert call() == binding.SD_ERR_ARG
    L.sd_cache_destroy(None)


def test_batch_tensors_are_checked():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        binding.CacheBatch(i32(2, 3), i32(3), i32(2), 2, 1)     # not on a GPU
    with pytest.raises(ValueError):
        binding.CacheBatch(i32(2, 3).long(), i32(3), i32(2), 2, 1)
    with pytest.raises(ValueError):
        binding.PagedCache(1, 1, 1, 64, 16, 1, 1, 1, dtype="fp8")


def test_index_arithmetic_stays_in_bounds(tmp_path):
    # the device functions that turn rows and positions into pool entries, run on the host over tables with bad entries
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "paging_host.cu")
    exe = str(tmp_path / "paging_host")
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, src], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok")


def test_plain_quantisation_by_exhaustive_search():
    g = torch.Generator().manual_seed(1)
    for dtype in ("int8", "e4m3"):
        values = torch.arange(-127, 128).double() if dtype == "int8" else torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double()
        values = values[~torch.isnan(values)].unique()
        x = torch.randn(50, 32, generator=g)
        codes, scale = P.quantise(x, dtype)
        near = (values.view(1, 1, -1) - (x.double() / scale.double().unsqueeze(1)).unsqueeze(2)).abs()
        assert torch.equal((codes.unsqueeze(2) - x.double().unsqueeze(2) / scale.double().view(-1, 1, 1)).abs().squeeze(2), near.min(2).values)
        assert float(codes.abs().max()) == P.TOP[dtype]


def test_plain_selection_against_direct_enumeration():
    g = torch.Generator().manual_seed(2)
    for trial in range(300):
        n = int(torch.randint(1, 9, (1,), generator=g))
        x = torch.randint(-3, 4, (n,), generator=g).float() * 0.7
        T, k, p, mp, u = float(torch.rand(1, generator=g)) + 0.2, trial % 5, [1.0, 0.6, 0.3][trial % 3], [0.0, 0.2][trial % 2], float(torch.rand(1, generator=g))
        order = sorted(range(n), key=lambda i: (-float(x[i]), i))
        w = [torch.exp((x[i].double() - x.max().double()) / T).item() for i in order]
        keep = len(w) if k == 0 else min(k, n)
        total = sum(w[:keep])
        run, kept = 0.0, []
        for i in range(keep):
            if p < 1 and i and run >= p * total:
                break
            if mp and i and w[i] < mp:
                break
            kept.append(i)
            run += w[i]
        target, run, want = u * run, 0.0, kept[-1]
        for i in kept:
            run += w[i]
            if run > target:
                want = i
                break
        assert P.select(x, u, T, k, p, mp) == order[want]


def test_threads_that_share_a_cache_hand_over_their_own_tensors(monkeypatch):
    # the library's call is replaced by a function that looks at the pointers it is given; layer names the thread
    from types import SimpleNamespace
    import sys
    import threading
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)
    tensors = [(torch.zeros(2, 3, 4), torch.zeros(2, 3, 4)) for _ in range(4)]
    wrong, calls = [], []

    @C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p)
    def append(h, layer, batch, k, v):
        got = tuple(binding.SdHeads.from_address(p).data for p in (k, v))
        calls.append(layer)
        if got != tuple(t.data_ptr() for t in tensors[layer]):
            wrong.append((layer, got))
        return binding.SD_OK

    cache = object.__new__(binding.PagedCache)
    cache.h, cache._append, cache._index, cache._raw, cache.device = None, append, -1, 0, "cpu"
    cache._kv_heads, cache._head_dim = 3, 4
    cache._described = binding._Described()
    batch = SimpleNamespace(n_tokens=2, index=-1, ref=0)

    def work(i):
        for _ in range(3000):
            cache.append(i, *tensors[i], batch)

    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    assert len(calls) == 12000
    assert not wrong, (len(wrong), wrong[0])


def test_options_of_a_cache_are_checked():
    L = binding.lib()
    assert L.sd_cache_set_option(None, binding.SD_CACHE_OPT_TEST_WAIT_EXPIRY, 1) == binding.SD_ERR_ARG
