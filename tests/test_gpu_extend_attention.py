"""The model over a paged cache with weights that make its logits depend on the attention: query and key products sixteen times as large
and the attention's share of the residual four times as large as in the plain random weights, whose scores are nearly equal.  Ignoring
the scores then moves the logits by fifteen times the tolerance and more (checked here, with the oracle), where it moves those of the plain
weights by less than it.  Tolerances are those of the other parity tests.

Over an 8-bit cache the oracle is given the keys and values that the cache holds, each checked to be within the largest code's step of its own: the
library's activations are fp16, so codes near a border come out one step apart, which by itself (emulated in the oracle) moves these logits
by up to 0.08 in e4m3."""
import pytest
import torch

import harness
import paged_reference as P
from oracle import skipdecode_oracle as O
from paper_2307_02628_b200 import binding, synth

pytestmark = pytest.mark.gpu

SHAPES = {64: synth.ModelShape("attending-64", 3, 256, 4, 512, 1000, 512, "bf16"), 128: synth.ModelShape("attending-128", 2, 512, 4, 512, 640, 512, "bf16"),
          32: synth.ModelShape("attending-32", 2, 64, 2, 128, 500, 512, "fp32")}


def attending_weights(shape, seed):
    w = synth.make_weights(shape, seed=seed)
    for layer in w["layers"]:
        layer["w_qkv"][:2 * shape.d_model] *= 4                 # powers of two: exact in bf16
        layer["w_o"] *= 4
    return w


def oracle(shape, w, seq, monkeypatch, change=lambda x, which: x):
    """Logits of every position; change is applied to the queries (1), keys (2) and values (0) of every layer."""
    calls = [0]
    split = O._split_heads

    def held(t, heads):
        calls[0] += 1
        return change(split(t, heads), calls[0] % 3)
    with monkeypatch.context() as m:
        m.setattr(O, "_split_heads", held)
        act = torch.ones(len(seq), shape.n_layers, dtype=torch.bool)
        return O.forward_sequence(w, shape.n_heads, seq.unsqueeze(0), act, torch.float64, logits_from=0)[0]


def page_table(n_tokens, page_len, seed):
    n = (n_tokens + page_len - 1) // page_len
    return torch.randperm(n + 2, generator=torch.Generator().manual_seed(seed))[:n].to(torch.int32).unsqueeze(0), n + 2


@pytest.mark.parametrize("hd,cache_dtype", [(32, "fp32"), (64, "bf16"), (128, "bf16"), (64, "int8"), (128, "e4m3")])
def test_one_sequence_in_chunks(hd, cache_dtype, monkeypatch):
    # the product that follows the attention is launched to begin early, and with one sequence follows the kernel for chunks itself
    shape = SHAPES[hd]
    w = attending_weights(shape, 5)
    chunks = [300, 1, 60, 45, 1, 90]
    seq = synth.make_tokens(shape.vocab, 1, sum(chunks), 40)[0]
    tol = harness.TOL["fp32" if cache_dtype == "fp32" else "bf16"]
    pages, n_pages = page_table(sum(chunks), 16, 1)
    dec = binding.Decoder(shape, w, 1, 300, 16)
    dec.set_option(binding.SD_OPT_DETERMINISTIC, 1)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, hd, 16, n_pages, 1, 512, cache_dtype, stream=dec.stream)
    at, got = 0, {}
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    for n in chunks:
        at += n
        b = binding.CacheBatch(pages.cuda(), i32([0, n]), i32([at]), n, n, at)
        ids = seq[at - n:at].cuda()
        one = dec.extend(cache, b, ids)
        for _ in range(10):                                     # the same tokens in the same places: the same bits
            assert torch.equal(dec.extend(cache, b, ids), one)
        got[at - 1] = one.cpu().double()[0]
    whole = binding.CacheBatch(pages.cuda(), i32([0, at]), i32([at]), at, at, at)
    held = [cache.read(l, whole) for l in range(shape.n_layers)]
    held = [{2: k.cpu().double().transpose(0, 1), 0: v.cpu().double().transpose(0, 1)} for k, v in held]
    layer_of = [0]

    def as_held(x, which):
        if which == 1:
            layer_of[0] += 1
            return x
        have = held[layer_of[0] - 1][which].unsqueeze(0)
        # the step of the largest code: the library's x differs from this one by a part of the row's size, not of each element's
        step = x.abs().amax(-1, keepdim=True) * (1 / 127 if cache_dtype == "int8" else 32 / 448)
        assert bool(((have - x).abs() <= step).all())
        return have
    ref = oracle(shape, w, seq, monkeypatch, as_held if cache_dtype in P.TOP else lambda x, which: x)
    blind = oracle(shape, w, seq, monkeypatch, lambda x, which: x * 0 if which == 1 else x)
    assert min(float((blind[p] - ref[p]).abs().max()) for p in got) > 15 * tol
    worst = max(float((lg - ref[p]).abs().max()) for p, lg in got.items())
    print(f"{shape.name} {cache_dtype}: max |err| {worst:.2e}")
    assert worst <= tol, worst
    assert dec.status() == 0 and cache.status() == 0
    cache.close()
    dec.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_one_sequence_captured(hd):
    shape = SHAPES[hd]
    dec = binding.Decoder(shape, attending_weights(shape, 6), 1, 300, 16)
    dec.set_option(binding.SD_OPT_DETERMINISTIC, 1)
    pages, n_pages = page_table(300, 32, 2)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, hd, 32, n_pages, 1, 512, "bf16", stream=dec.stream)
    b = binding.CacheBatch(pages.cuda(), torch.tensor([0, 300], dtype=torch.int32).cuda(), torch.tensor([300], dtype=torch.int32).cuda(), 300, 300, 300)
    ids = synth.make_tokens(shape.vocab, 1, 300, 3)[0].to(torch.int32).cuda()
    want = dec.extend(cache, b, ids)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    with torch.cuda.stream(dec.stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=dec.stream):
            dec.extend(cache, b, ids, logits=out)
        for _ in range(50):
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)
    assert dec.status() == 0 and cache.status() == 0
    cache.close()
    dec.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_prompts_agree_with_prefill(hd, monkeypatch):
    # both keep 16 bits of queries and weights over the same bf16 keys and values
    shape = SHAPES[hd]
    w = attending_weights(shape, 7)
    prompts = synth.make_tokens(shape.vocab, 3, 300, 9)
    wl = synth.Workload(shape, 3, 300, 4, shape.n_layers, shape.n_layers, 0)
    dec = harness.make_decoder(wl, w)
    dec.schedule(shape.n_layers, shape.n_layers, 0, wl.gen_len)
    pages = torch.randperm(3 * 19, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(3, 19)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, hd, 16, 3 * 19, 3, 900, "bf16", stream=dec.stream)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    with torch.cuda.stream(dec.stream):
        a = dec.prefill(prompts).clone()
        b = dec.extend(cache, binding.CacheBatch(pages.cuda(), i32([0, 300, 600, 900]), i32([300] * 3), 900, 300, 300), prompts.reshape(-1))
    dec.synchronize()
    ref = torch.stack([oracle(shape, w, p, monkeypatch)[-1] for p in prompts])
    far = [float((x.cpu().double() - ref).abs().max()) for x in (a, b)]
    print(f"{shape.name}: prefill {far[0]:.2e}, extend {far[1]:.2e}, apart {float((a - b).abs().max()):.2e}")
    assert max(far) <= harness.TOL["bf16"]
    assert dec.status() == 0 and cache.status() == 0
    cache.close()
    dec.close()
