"""CPU-only checks of attention with changed scores: refusals, the mask's index arithmetic, the limits that the GPU tests use."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paged_bounds as B
import paged_reference as P
import scores_reference as S
from paper_2307_02628_b200 import binding, build


def test_null_arguments_are_refused():
    L = binding.lib()
    b, r, s = binding.SdBatch(), binding.SdHeads(), binding.SdScores()
    assert L.sd_cache_attention_scores(None, 0, C.byref(b), C.byref(r), 0.0, C.byref(s), C.byref(r)) == binding.SD_ERR_ARG


def test_tensors_are_checked():
    with pytest.raises(ValueError):
        binding.Scores(slopes=torch.zeros(4))                  # not on a GPU
    with pytest.raises(ValueError):
        binding.Scores(lo=torch.zeros(4, dtype=torch.int32))
    assert binding.Scores(cap=3.0, window=5).c.window == 5


def test_what_a_row_sees_stays_in_its_sequence(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "scores_host.cu")
    exe = str(tmp_path / "scores_host")
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, src], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok")


def test_without_changes_the_reference_is_the_plain_one():
    lay = P.Layout([1, 20, 5], [50, 20, 3], 16, seed=1)
    contents = B.contents_of(lay, 2, 64, 2)
    q = torch.randn(lay.n_tokens, 4, 64, generator=torch.Generator().manual_seed(3))
    for a, b in zip(S.reference(q, contents, lay, 0.125, 2), B.reference(q, contents, lay, 0.125, 2)):
        assert torch.equal(a, b)


def test_the_limit_notices_a_wrong_mask_cap_or_slope():
    """A key too many or too few, a slope or a cap that is off by a hundredth, in a row of 60 keys."""
    lay = P.Layout([30], [90], 16, seed=1)
    contents = B.contents_of(lay, 2, 64, 2)
    q = 3 * torch.randn(30, 4, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    slopes = torch.tensor([0.5, 0.25, 0.1, 0.05])
    right = dict(cap=6.0, slopes=slopes, window=40)
    out = S.reference(q, contents, lay, 0.125, 2, **right)
    for wrong in (dict(right, window=41), dict(right, window=39), dict(right, cap=6.1), dict(right, slopes=slopes * 1.02)):
        got = S.reference(q, contents, lay, 0.125, 2, **wrong)[0].bfloat16()
        assert float(S.over(got, *out, 64, q.dtype, 6.0).max()) > 1, wrong
    assert float(S.over(out[0].bfloat16(), *out, 64, q.dtype, 6.0).max()) < 1


@pytest.mark.parametrize("bad", [dict(window=2 ** 32), dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(window=-(2 ** 31) - 1), dict(window=0.5), dict(window=2.5), dict(window=float("inf")), dict(window=float("nan")),
                                 dict(cap=1e-46), dict(cap=-1e-50)])
def test_numbers_that_would_arrive_as_others_are_refused(bad):
    """A window of 2^32 would be none, a cap of 1e-46 off: the library sees 32 bits of either."""
    with pytest.raises(ValueError):
        binding.Scores(**bad)


def test_numbers_that_arrive_as_they_are():
    for kw in (dict(window=2 ** 31 - 1), dict(window=-1), dict(window=2048.0), dict(cap=0.0), dict(cap=1e-35), dict(cap=float("inf")), dict(cap=-1.0)):
        c = binding.Scores(**kw).c                             # what is out of its range is the library's to refuse
        for name, value in kw.items():
            assert getattr(c, name) == pytest.approx(value, rel=2.0 ** -24, abs=0)
