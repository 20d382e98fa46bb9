"""The model over a paged cache (sd_extend): prompts in one piece and in chunks, single tokens under a layer budget, sequences at
positions of their own, against the oracle.  Tolerances are those of the other parity tests (1e-4 in fp32, 3e-2 in bf16 storage).

With an 8-bit cache the oracle is given the same cache: its keys and values are rounded to the codes the definition gives.  The
library's fp32 keys differ from the oracle's in the last bits, so a code next to a border can land one step away: one of
127 steps of a head's largest element, in a few elements, which moves a logit by far less than the storage tolerance.
"""
import pytest
import torch

import harness
import paged_reference as P
from oracle import skipdecode_oracle as O
from paper_2307_02628_b200 import binding, synth

pytestmark = pytest.mark.gpu

BF16 = synth.ModelShape("extend-bf16", 3, 256, 4, 512, 1000, 256, "bf16")
WIDE = synth.ModelShape("extend-wide", 2, 512, 4, 512, 640, 256, "bf16")      # head size 128
FP32 = synth.TINY


class Pages:
    """Hands out the pages of a cache; the table lives on the device."""

    def __init__(self, n_seqs, columns, n_pages, page_len, seed=0):
        self.free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = torch.full((n_seqs, columns), -1, dtype=torch.int32)
        self.len = [0] * n_seqs
        self.page_len = page_len

    def grow(self, new):
        """Sequences that take new[s] more tokens: (first, max_new) and the batch for the device."""
        first = [0]
        for s, n in enumerate(new):
            for p in range(self.len[s], self.len[s] + n):
                if p % self.page_len == 0:
                    self.table[s, p // self.page_len] = self.free.pop()
            self.len[s] += n
            first.append(first[-1] + n)
        return binding.CacheBatch(self.table.cuda(), torch.tensor(first, dtype=torch.int32).cuda(), torch.tensor(self.len, dtype=torch.int32).cuda(),
                                  first[-1], max(new))


def oracle_logits(shape, w, seq, act, cache_dtype=None, monkeypatch=None):
    """Logits of every position of one sequence whose position t runs the layers act[t]."""
    if cache_dtype in P.TOP:
        split = O._split_heads

        def held(t, H, _n=[0]):
            out = split(t, H)
            _n[0] += 1
            return out if _n[0] % 3 == 1 else P.stored(out.float(), cache_dtype).double()      # called for q, k, v in turn
        monkeypatch.setattr(O, "_split_heads", held)
    out = O.forward_sequence(w, shape.n_heads, seq.unsqueeze(0), act, torch.float64, logits_from=0)[0]
    if cache_dtype in P.TOP:
        monkeypatch.setattr(O, "_split_heads", split)
    return out


@pytest.mark.parametrize("shape,cache_dtype", [(FP32, "fp32"), (FP32, "bf16"), (BF16, "bf16"), (BF16, "fp32"), (WIDE, "bf16"),
                                               (BF16, "int8"), (WIDE, "int8"), (WIDE, "e4m3")], ids=lambda x: getattr(x, "name", x))
def test_chunks_and_steps_match_the_oracle(shape, cache_dtype, monkeypatch):
    w = synth.make_weights(shape, seed=5)
    n_seqs, page = 3, 16
    total = [61, 90, 34]                                        # prompt tokens of each sequence
    tokens = [synth.make_tokens(shape.vocab, 1, t + 8, 40 + s)[0] for s, t in enumerate(total)]
    dec = binding.Decoder(shape, w, n_seqs, 90, 16)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, shape.head_dim, page, 24, n_seqs, 256, cache_dtype, stream=dec.stream)
    pages = Pages(n_seqs, 8, 24, page)
    tol = harness.TOL["fp32" if shape.dtype == "fp32" and cache_dtype == "fp32" else "bf16"]
    L = shape.n_layers
    # chunks of different sizes, some sequences sitting a call out; then single tokens, the budget falling to L - 1 layers (1 of
    # warm-up) and, where there are three, to L - 2
    plan = [([61, 7, 0], L), ([0, 40, 33], L), ([0, 43, 1], L)] + [([1, 1, 1], L)] * 2 + [([1, 1, 1], L - 1)] * 3 + [([1, 0, 1], max(L - 2, 2 if L > 2 else 1))] * 2
    warmup = 1 if L > 2 else 0
    act = [[] for _ in range(n_seqs)]
    got = [dict() for _ in range(n_seqs)]
    for new, n in plan:
        begin = list(pages.len)
        b = pages.grow(new)
        ids = torch.cat([tokens[s][begin[s]:begin[s] + new[s]] for s in range(n_seqs)])
        logits = dec.extend(cache, b, ids, n, warmup).cpu()
        for s in range(n_seqs):
            layers = [l < warmup or l >= L - (n - warmup) for l in range(L)]
            act[s] += [layers] * new[s]
            if new[s]:
                got[s][pages.len[s] - 1] = logits[s]
    assert cache.status() == 0 and dec.status() == 0
    worst = 0.0
    for s in range(n_seqs):
        seq = tokens[s][:pages.len[s]]
        a = torch.tensor(act[s])
        kw = {}
        ref = oracle_logits(shape, w, seq, a, cache_dtype, monkeypatch)
        for p, lg in got[s].items():
            worst = max(worst, float((lg.double() - ref[p]).abs().max()))
            assert float(ref[p].abs().max()) > 0.05
    print(f"{shape.name} {cache_dtype}: max |err| {worst:.2e}")
    assert worst <= tol, worst
    cache.close()
    dec.close()


@pytest.mark.parametrize("cache_dtype", ["bf16", "int8"])
def test_a_whole_serving_run_graphed_and_sampled(cache_dtype):
    """Prompt chunks, then decode steps whose append, attention and selection are replayed from one graph: the same tokens as the
    same calls made one by one."""
    shape, n_seqs, page, steps = BF16, 4, 16, 20
    w = synth.make_weights(shape, seed=6)
    dec = binding.Decoder(shape, w, n_seqs, 64, 64)
    dec.set_option(binding.SD_OPT_DETERMINISTIC, 1)
    settings = dict(temperature=torch.tensor([0.3, 0.7, 1.0, 0.0]).cuda(), top_k=torch.tensor([0, 40, 0, 0], dtype=torch.int32).cuda(),
                    top_p=torch.tensor([0.7, 0.9, 1.0, 1.0]).cuda(), min_p=torch.tensor([0.0, 0.02, 0.0, 0.0]).cuda())
    prompts = [synth.make_tokens(shape.vocab, 1, 20 + 9 * s, 7 + s)[0] for s in range(n_seqs)]
    uniforms = synth.make_uniforms(n_seqs * (steps + 1), 3).view(-1, n_seqs).cuda()

    def serve(graphed):
        cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, shape.head_dim, page, 40, n_seqs, 256, cache_dtype, stream=dec.stream)
        pages = Pages(n_seqs, 8, 40, page)
        out = []
        with torch.cuda.stream(dec.stream):
            b = pages.grow([len(p) for p in prompts])
            logits = dec.extend(cache, b, torch.cat(prompts))
            ids = dec.sample(logits, uniforms[0], **settings)
            # the tables for all steps are handed out ahead; the lengths grow on the device
            b = pages.grow([steps] * n_seqs)
            length = torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda()
            one = binding.CacheBatch(b.pages, torch.arange(n_seqs + 1, dtype=torch.int32).cuda(), length, n_seqs, 1, 96)
            logits = torch.zeros_like(logits)
            u = torch.zeros(n_seqs, device="cuda")
            graph = None
            for t in range(steps):
                out.append(ids.clone())
                u.copy_(uniforms[t + 1])
                length += 1
                if graphed and t == 1:
                    graph = torch.cuda.CUDAGraph()
                    torch.cuda.synchronize()
                    with torch.cuda.graph(graph, stream=dec.stream):
                        dec.extend(cache, one, ids, shape.n_layers - 1, 0, logits)
                        dec.sample(logits, u, out=ids, **settings)
                if graph is not None:
                    graph.replay()
                else:
                    dec.extend(cache, one, ids, shape.n_layers - 1, 0, logits)
                    dec.sample(logits, u, out=ids, **settings)
            out.append(ids.clone())
            dec.stream.synchronize()
        assert cache.status() == 0 and dec.status() == 0
        cache.close()
        return torch.stack(out).cpu()

    a, b = serve(False), serve(True)
    assert torch.equal(a, b)
    assert len(set(a[:, 2].tolist())) > 3                       # a run that chooses, not one token over and over
    dec.close()


def test_extend_agrees_with_prefill_and_decode_step():
    shape = WIDE
    wl = synth.Workload(shape, 5, 40, 6, shape.n_layers, 1, 0)
    w = synth.make_weights(shape, seed=8)
    dec = harness.make_decoder(wl, w)
    prompts, forced = synth.make_prompts(wl), synth.make_forced_tokens(wl)
    cache = binding.PagedCache(shape.n_layers, shape.n_heads, shape.n_heads, shape.head_dim, 32, 16, 5, 256, "bf16", stream=dec.stream)
    pages = Pages(5, 4, 16, 32)
    with torch.cuda.stream(dec.stream):                         # prefill and decode_step leave their results to the handle's stream
        n_active, _ = dec.schedule(wl.max_layers, wl.min_layers, 0, wl.gen_len)
        a = [dec.prefill(prompts).clone()]
        b = [dec.extend(cache, pages.grow([40] * 5), prompts.reshape(-1))]
        for g in range(wl.gen_len):
            ids = forced[:, g].contiguous()
            b.append(dec.extend(cache, pages.grow([1] * 5), ids, n_active[g]))
            a.append(dec.decode_step(ids, 40 + g).clone())      # the two do not disturb each other
    dec.synchronize()
    for x, y in zip(a, b):
        assert float((x - y).abs().max()) <= 2 * harness.TOL["bf16"]      # each is within the tolerance of the same oracle
    cache.close()
    dec.close()


def test_refusals():
    shape = BF16
    dec = binding.Decoder(shape, synth.make_weights(shape, seed=1), 2, 16, 8)
    mk = lambda **k: binding.PagedCache(**{**dict(n_layers=3, n_heads=4, n_kv_heads=4, head_dim=64, page_len=16, n_pages=8, max_seqs=4,  # noqa: E731
                                                  max_tokens=8192, dtype="bf16", stream=dec.stream), **k})
    pages = Pages(2, 4, 8, 16)
    b = pages.grow([3, 2])
    ids = torch.zeros(5, dtype=torch.int32)
    good = mk()
    for cache, args, code in ((mk(n_layers=2), (), binding.SD_ERR_ARG), (mk(n_kv_heads=2), (), binding.SD_ERR_ARG), (mk(head_dim=32), (), binding.SD_ERR_ARG),
                              (mk(stream=torch.cuda.Stream()), (), binding.SD_ERR_ARG), (good, (0, 0), binding.SD_ERR_ARG),
                              (good, (4, 0), binding.SD_ERR_ARG), (good, (2, 2), binding.SD_ERR_ARG), (good, (2, -1), binding.SD_ERR_ARG)):
        with pytest.raises(binding.SdError) as e:
            dec.extend(cache, b, ids, *args)
        assert e.value.code == code
    with pytest.raises(ValueError):
        dec.extend(good, b, ids[:4])
    three = Pages(3, 4, 8, 16).grow([1, 1, 1])                  # more sequences than the handle's batch
    with pytest.raises(binding.SdError) as e:
        dec.extend(good, three, ids[:3])
    assert e.value.code == binding.SD_ERR_CAPACITY
    many = binding.CacheBatch(b.pages, b.first, b.length, 4097, 4097)
    with pytest.raises(binding.SdError) as e:
        dec.extend(good, many, torch.zeros(4097, dtype=torch.int32))
    assert e.value.code == binding.SD_ERR_CAPACITY
    dec.extend(good, b, ids)
    assert dec.status() == 0 and good.status() == 0
    # a token id out of range is reported as in the decode step
    dec.extend(good, b, ids + shape.vocab)
    assert dec.status() == binding.STATUS_BAD_TOKEN
    dec.close()


def test_tensors_elsewhere_are_refused_and_launches_are_counted():
    shape = BF16
    dec = binding.Decoder(shape, synth.make_weights(shape, seed=1), 2, 16, 8)
    cache = binding.PagedCache(3, 4, 4, 64, 16, 8, 4, 64, dtype="bf16", stream=dec.stream)
    b = Pages(2, 4, 8, 16).grow([3, 2])
    ids = torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError):
        dec.extend(cache, b, ids, logits=torch.empty(2, shape.vocab))              # host memory
    dec.extend(cache, b, ids)
    n0 = dec.launch_count()
    dec.extend(cache, b, ids)
    # rows, embedding; per layer two LayerNorms, four products, append, attention; LayerNorm and LM head
    assert dec.launch_count() - n0 == 2 + 3 * 8 + 2
    dec.extend(cache, b, ids, n_active=2)
    assert dec.launch_count() - n0 == 2 * (2 + 2) + (3 + 2) * 8
    assert dec.status() == 0 and cache.status() == 0
    cache.close()
    dec.close()
