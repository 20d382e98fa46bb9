"""A model on a paged cache in 4 bits (sd_extend): prompts in chunks and single tokens against the oracle.

The oracle attends to what the cache holds, read back from it, so that logits are held to the tolerances of the other parity tests.  What
the cache holds is held to the oracle's own keys and values: a code is off by at most half of its largest step, 1, and by 0.375 more where
the block scale (4 bits, off by at most 2^-4 of itself) came out too small for the block's largest element, in units of block scale times
scale; 3e-2 on top, the tolerance of a 16-bit model's hidden states.
"""
import pytest
import torch

import harness
from oracle import skipdecode_oracle as O
from paper_2307_02628_b200 import binding, synth

pytestmark = pytest.mark.gpu

BF16 = synth.ModelShape("four-bf16", 3, 256, 4, 512, 1000, 256, "bf16")
WIDE = synth.ModelShape("four-wide", 2, 512, 4, 512, 640, 256, "bf16")      # head size 128


@pytest.mark.parametrize("shape", [synth.TINY, BF16, WIDE], ids=lambda s: s.name)
def test_chunks_and_steps_match_the_oracle(shape, monkeypatch):
    w = synth.make_weights(shape, seed=5)
    total, page, columns = [61, 90, 34], 16, 6
    tokens = [synth.make_tokens(shape.vocab, 1, t, 40 + s)[0] for s, t in enumerate(total)]
    dec = binding.Decoder(shape, w, 3, 90, 16)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, shape.head_dim, page, 18, 3, 256, "e2m1", stream=dec.stream)
    table = torch.randperm(18, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(3, columns).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    begin, got = [0, 0, 0], [dict() for _ in total]
    for new in ([40, 7, 0], [19, 70, 31], [1, 1, 1], [0, 12, 2], [1, 0, 0]):
        end = [b + n for b, n in zip(begin, new)]
        first = [0, new[0], new[0] + new[1], sum(new)]
        ids = torch.cat([tokens[s][begin[s]:end[s]] for s in range(3)])
        logits = dec.extend(cache, binding.CacheBatch(table, i32(first), i32(end), sum(new), max(new)), ids).cpu()
        for s in range(3):
            if new[s]:
                got[s][end[s] - 1] = logits[s].double()
        begin = end
    assert begin == total and cache.status() == 0 and dec.status() == 0
    whole = binding.CacheBatch(table, i32([0, 61, 151, 185]), i32(total), 185, 90)
    held = [[t.cpu().double().transpose(0, 1) for t in cache.read(l, whole)] for l in range(shape.n_layers)]
    units = []
    for l in range(shape.n_layers):                              # block scale times scale of every element
        pool = cache.layer(l)
        at = torch.cat([torch.stack((table[s, torch.arange(n) // page].cpu().long(), torch.arange(n) % page)) for s, n in enumerate(total)], 1).cuda()
        units.append([(pool[n + "_block"].float() * pool[n + "_scale"].unsqueeze(-1))[at[0], :, at[1]].repeat_interleave(16, -1).cpu().double().transpose(0, 1)
                      for n in ("k", "v")])
    split = O._split_heads
    tol = harness.TOL["bf16" if shape.dtype == "bf16" else "fp32"]
    for s, n in enumerate(total):
        rows = slice(sum(total[:s]), sum(total[:s + 1]))
        calls, far = [0], []

        def from_cache(t, H):
            out = split(t, H)
            layer, which = divmod(calls[0], 3)                   # called for q, k, v in turn
            calls[0] += 1
            if which == 0:
                return out
            far.append(float(((held[layer][which - 1][:, rows] - out[0]).abs() - 1.375 * units[layer][which - 1][:, rows]).max()))
            return held[layer][which - 1][:, rows].unsqueeze(0)
        monkeypatch.setattr(O, "_split_heads", from_cache)
        ref = O.forward_sequence(w, shape.n_heads, tokens[s].unsqueeze(0), torch.ones(n, shape.n_layers, dtype=torch.bool), torch.float64, logits_from=0)[0]
        monkeypatch.setattr(O, "_split_heads", split)
        assert len(far) == 2 * shape.n_layers and max(far) <= 3e-2, far
        for p, lg in got[s].items():
            assert float(ref[p].abs().max()) > 0.05
            assert float((lg - ref[p]).abs().max()) <= tol, (s, p)
    cache.close()
    dec.close()
