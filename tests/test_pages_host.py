"""CPU-only checks of the calls on pages: refusals, the index arithmetic that the kernels share, the plain form that the GPU tests compare with."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

import pages_reference as R
from paper_2307_02628_b200 import binding, build


def test_null_arguments_are_refused():
    L = binding.lib()
    t = binding.SdTables()
    for call in (lambda: L.sd_cache_fork(None, C.byref(t), 1, 1, 1), lambda: L.sd_cache_resize(None, C.byref(t), 1),
                 lambda: L.sd_cache_compact(None, C.byref(t), None), lambda: L.sd_cache_copy(None, 1, 1, 1)):
        assert call() == binding.SD_ERR_ARG


def test_tables_are_checked():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        binding.PageTables(i32(2, 3), i32(2), i32(5))          # not on a GPU


def test_index_arithmetic_stays_in_bounds(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "pages_host.cu")
    exe = str(tmp_path / "pages_host")
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, src], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok")


def test_plain_form_keeps_its_books():
    for seed in range(40):
        r = random.Random(seed)
        books = R.Books(12, 9, r.choice([40, 100]), r.choice([8, 16]))
        for _ in range(30):
            what = r.random()
            if what < 0.6:
                books.resize(R.random_targets(books, r, books.page_len * 8))
            elif what < 0.8:
                empty = [s for s, n in enumerate(books.len) if n == 0]
                r.shuffle(empty)
                live = [s for s, n in enumerate(books.len) if n]
                if live:
                    books.fork([r.choice(live) for _ in empty[:3]], empty[:3])
            else:
                copies, used = books.compact()
                assert all(books.refs[:used]) and not any(books.refs[used:])
                assert not {f for f, _ in copies} & {t for _, t in copies}
            books.check()
