"""Attention over a paged cache in 4 bits held to the limits that one missing key exceeds (see paged_bounds): tiles' borders, split keys, types of queries
and results, pages that do not exist."""
import pytest

from test_gpu_scores import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,heads,page", [(64, 4, 16), (64, 4, 128), (128, 7, 64), (128, 4, 8)])
def test_split_keys(hd, heads, page):
    run("e2m1", heads, 1, hd, page, [100, 40, 300, 9], [2900, 2049, 300, 4], seed=hd, start=2, tail=1, plain=True)
    run("e2m1", heads, 1, hd, page, [65], [3333], seed=hd + 1, plain=True)
    run("e2m1", heads, 1, hd, page, [33, 8], [4097, 2560], seed=hd + 2, max_len=1500, plain=True)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,length", [([128], [128]), ([127], [255]), ([129], [129]), ([256, 1], [513, 511]), ([300], [700]), ([64, 257], [64, 258]),
                                         ([65, 130, 191], [193, 320, 191])])
def test_borders_of_tiles(hd, new, length):
    for page in (8, 32, 128):
        run("e2m1", 2, 2, hd, page, new, length, seed=sum(new) + page, plain=True)


@pytest.mark.parametrize("io,out_dtype", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "bf16"), ("fp16", "bf16")])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_types(io, out_dtype, hd):
    run("e2m1", 4, 2, hd, 16, [1, 70, 9], [40, 300, 9], io=io, out_dtype=out_dtype, seed=hd, plain=True)
    run("e2m1", 4, 2, hd, 64, [130], [1000], io=io, out_dtype=out_dtype, seed=hd, k_gain=3.0, scale=-0.1, plain=True)


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_pages_that_do_not_exist(hd):
    run("e2m1", 2, 2, hd, 16, [90, 1, 3], [300, 200, 20], seed=3, gone=((0, 3), (0, 4), (1, 0), (2, 1), (1, 12)), plain=True)
