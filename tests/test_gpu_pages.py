"""Forking, resizing, compacting and copying pages of a paged cache: books and contents equal to the plain form's."""
import random

import pytest
import torch

import pages_reference as R
from paper_2307_02628_b200 import binding, synth

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


class Both:
    """A cache with random contents, its books on the device, and their plain form."""

    def __init__(self, n_seqs, columns, n_pages, page_len, dtype="bf16", layers=2, kv_heads=2, hd=32, seed=0, max_seqs=None):
        self.cache = binding.PagedCache(layers, kv_heads, kv_heads, hd, page_len, n_pages, max_seqs or n_seqs, 8, dtype)
        self.books = R.Books(n_seqs, columns, n_pages, page_len)
        self.tables = binding.PageTables.empty(self.cache, n_seqs, columns)
        self.layers = layers
        g = torch.Generator(device="cuda").manual_seed(seed)
        for pool in self.pools():
            pool.copy_(torch.randint(0, 256, pool.shape, generator=g, device="cuda", dtype=torch.uint8))
        self.want = [p.clone() for p in self.pools()]

    def pools(self):
        return [t.view(torch.uint8).flatten(1) for l in range(self.layers) for t in self.cache.layer(l).values()]

    def push(self):
        self.tables.pages.copy_(i32(self.books.pages))
        self.tables.length.copy_(i32(self.books.len))
        self.tables.refs.copy_(i32(self.books.refs))

    def copied(self, copies):
        if copies:
            f, t = (torch.tensor(x).cuda() for x in zip(*copies))
            for p in self.want:
                p[t] = p[f]

    def same(self, status=0):
        assert self.cache.status() == status
        b = self.books
        assert self.tables.length.cpu().tolist() == b.len
        assert self.tables.refs.cpu().tolist() == b.refs
        pages = self.tables.pages.cpu()
        for s, row in enumerate(b.pages):
            n = b.used_columns(b.len[s])
            assert pages[s, :n].tolist() == row[:n], s
        for got, want in zip(self.pools(), self.want):
            assert torch.equal(got, want)

    def fork(self, src, dst):
        self.copied(self.books.fork(src, dst))
        self.cache.fork(self.tables, i32(src), i32(dst))

    def resize(self, target):
        self.copied(self.books.resize(target))
        self.cache.resize(self.tables, i32(target))

    def compact(self):
        copies, used = self.books.compact()
        self.copied(copies)
        assert self.cache.compact(self.tables).tolist() == [used]


@pytest.mark.parametrize("dtype,kv_heads,hd,page_len", [("fp32", 1, 32, 8), ("bf16", 3, 64, 16), ("int8", 2, 128, 32), ("e4m3", 1, 64, 128), ("e2m1", 1, 32, 8),
                                                       ("e2m1", 5, 128, 64), ("bf16", 12, 128, 64)])
def test_random_calls(dtype, kv_heads, hd, page_len):
    r = random.Random(hd + page_len)
    b = Both(13, 7, 60, page_len, dtype, kv_heads=kv_heads, hd=hd, seed=page_len)
    for step in range(40):
        b.books.short = False
        what = r.random()
        if what < 0.55:
            b.resize(R.random_targets(b.books, r, page_len * 7))
        elif what < 0.8:
            empty = [s for s, n in enumerate(b.books.len) if n == 0]
            live = [s for s, n in enumerate(b.books.len) if n]
            r.shuffle(empty)
            if live and empty:
                b.fork([r.choice(live) for _ in empty[:5]], empty[:5])
        else:
            b.compact()
        b.same(binding.STATUS_NO_PAGES if b.books.short else 0)


def test_pools_of_many_pages_and_many_rows():
    # more pages than a span of the search for free ones, more rows than threads
    r = random.Random(3)
    b = Both(2500, 12, 20011, 8, layers=1, kv_heads=1, seed=3)
    b.resize([r.randint(0, 70) for _ in range(2500)])
    b.same()
    b.resize([n if r.random() < 0.4 else 0 if r.random() < 0.5 else r.randint(0, 96) for n in b.books.len])
    b.same()
    empty, live = [s for s, n in enumerate(b.books.len) if n == 0], [s for s, n in enumerate(b.books.len) if n]
    b.fork([r.choice(live) for _ in empty], empty)
    b.same()
    b.books.check()
    b.compact()
    b.same()
    b.resize([0] * 2500)
    b.same()
    assert not any(b.books.refs)


def test_too_few_pages():
    b = Both(6, 8, 10, 8)
    b.resize([20, 16, 8, 0, 0, 0])                               # 3 + 2 + 1 pages, 4 left
    b.same()
    b.resize([24, 16, 8, 17, 16, 8])                             # the fifth is short of a page, and so is everybody behind it that needs one
    assert b.books.short and b.books.len == [24, 16, 8, 17, 0, 0]
    b.same(binding.STATUS_NO_PAGES)
    b.books.short = False
    b.resize([21, 16, 0, 17, 0, 0])
    b.same()
    b.fork([0, 3, 0], [2, 4, 5])                                 # two copies, two pages left: the third is short
    assert b.books.short and b.books.len[5] == 0
    b.same(binding.STATUS_NO_PAGES)
    b.books.short = False
    b.resize([21, 16, 16, 17, 17, 0])                            # a cut to whole pages needs none
    b.same()


def test_a_cut_inside_a_shared_page_gets_a_copy():
    b = Both(4, 8, 20, 16)
    b.resize([64, 0, 0, 0])
    b.fork([0, 0], [1, 2])
    b.same()
    b.resize([64, 50, 50, 0])                                    # both forks end inside the same shared page
    b.same()
    assert len({b.books.pages[s][3] for s in range(3)}) == 3
    b.resize([41, 64, 0, 0])                                     # the first one too, now that nobody shares: in place
    b.same()
    b.books.check()


def test_growing_inside_a_page_that_the_caller_shares():
    b = Both(2, 4, 8, 16)
    b.resize([10, 0])
    b.books.pages[1][0], b.books.len[1], b.books.refs[b.books.pages[0][0]] = b.books.pages[0][0], 10, 2
    b.push()
    b.resize([10, 10])                                           # as long as they were: both get pages of their own
    b.same()
    assert b.books.pages[0][0] != b.books.pages[1][0]


def test_wrong_calls_are_reported_and_skipped():
    bad = binding.STATUS_BAD_BATCH
    b = Both(5, 4, 12, 8)
    b.resize([10, 20, 0, 0, 0])
    b.same()
    # rows out of range, a row onto itself, onto one that is not empty, two onto one (the first one counts)
    b.cache.fork(b.tables, i32([9, 0, 1, 0, 1]), i32([2, -1, 1, 1, 3]))
    b.copied(b.books.fork([1], [3]))
    b.same(bad)
    b.cache.fork(b.tables, i32([0, 1]), i32([4, 4]))
    b.copied(b.books.fork([0], [4]))
    b.same(bad)
    # lengths out of range leave their rows alone
    b.cache.resize(b.tables, i32([33, -1, 8, 2 ** 31 - 1, 0]))
    b.copied(b.books.resize([b.books.len[0], b.books.len[1], 8, b.books.len[3], 0]))
    b.same(bad)
    # a page given back that nobody was said to hold, and entries that are no pages
    b.books.refs[b.books.pages[0][1]] = 0
    b.books.pages[1][2] = 77
    b.push()
    b.cache.resize(b.tables, i32([8, 10, 8, 20, 0]))
    assert b.cache.status() == bad
    assert int(b.tables.refs.min()) >= 0
    b.cache.copy_pages(i32([0, -1, 12, 3]), i32([11, 2, 3, 3]))
    b.want = [p.clone() for p in b.want]
    assert b.cache.status() == bad
    for got in b.pools():
        assert torch.equal(got[11], got[0])


def test_wrong_entries_are_not_followed_by_compaction_and_forks():
    bad = binding.STATUS_BAD_BATCH
    b = Both(4, 4, 16, 8)
    b.resize([8, 8, 8, 32])
    b.resize([8, 0, 8, 32])
    b.books.pages[0][0], b.books.pages[2][0] = 99, -5
    b.push()
    b.cache.fork(b.tables, i32([0]), i32([1]))
    assert b.cache.status() == bad and b.tables.pages[1, 0].item() == -1
    b.cache.compact(b.tables)
    assert b.cache.status() == bad
    assert b.tables.pages[0, 0].item() == 99 and b.tables.pages[2, 0].item() == -5


def test_copy_pages():
    for dtype in ("bf16", "e2m1"):
        b = Both(1, 1, 50, 16, dtype, layers=3, kv_heads=7, hd=64)
        order = torch.randperm(50, generator=torch.Generator().manual_seed(1)).tolist()
        src, dst = order[:20], order[20:40]
        b.copied(list(zip(src, dst)))
        b.cache.copy_pages(i32(src), i32(dst))
        b.cache.copy_pages(i32([]), i32([]))
        b.same()


def test_captured_calls_follow_the_books():
    stream = torch.cuda.Stream()
    b = Both(6, 6, 40, 8, seed=2)
    b.cache.close()
    b.cache = binding.PagedCache(2, 2, 2, 32, 8, 40, 6, 8, "bf16", stream=stream)
    for t in b.pools():
        t.fill_(3)
    for i, t in enumerate(b.pools()):
        t.copy_(torch.arange(40, device="cuda").to(torch.uint8).unsqueeze(1).expand_as(t) + i)
    b.want = [p.clone() for p in b.pools()]
    src, dst, target = i32([0, 1]), i32([4, 5]), i32([0] * 6)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.cache.resize(b.tables, target)
        b.cache.fork(b.tables, src, dst)
        used = b.cache.compact(b.tables)
    for targets in ([13, 20, 7, 0, 0, 0], [30, 9, 0, 16, 0, 0], [33, 33, 3, 1, 0, 0]):
        target.copy_(i32(targets))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.copied(b.books.resize(targets))
        b.copied(b.books.fork([0, 1], [4, 5]))
        copies, n = b.books.compact()
        b.copied(copies)
        assert used.tolist() == [n]
        b.same()
        b.books.check()


def test_refusals():
    b = Both(4, 4, 16, 8)
    L, h, t = binding.lib(), b.cache.h, b.tables
    x = i32([0, 1, 2, 3, 0])
    p = x.data_ptr()
    import ctypes as C
    wide = binding.SdTables(t.c.pages, t.c.len, t.c.refs, 5, 4)
    far = binding.SdTables(t.c.pages, t.c.len, t.c.refs, 4, 2 ** 27 + 1)
    none = binding.SdTables(t.c.pages, None, t.c.refs, 4, 4)
    empty = binding.SdTables(t.c.pages, t.c.len, t.c.refs, 0, 4)
    for code, tables in ((binding.SD_ERR_CAPACITY, wide), (binding.SD_ERR_ARG, far), (binding.SD_ERR_ARG, none), (binding.SD_ERR_ARG, empty)):
        assert L.sd_cache_fork(h, C.byref(tables), p, p, 1) == code
        assert L.sd_cache_resize(h, C.byref(tables), p) == code
        assert L.sd_cache_compact(h, C.byref(tables), None) == code
    assert L.sd_cache_fork(h, t.ref, p, p, 5) == binding.SD_ERR_ARG       # more forks than rows
    assert L.sd_cache_fork(h, t.ref, p, p, -1) == binding.SD_ERR_ARG
    assert L.sd_cache_fork(h, t.ref, None, p, 1) == binding.SD_ERR_ARG
    assert L.sd_cache_fork(h, t.ref, None, None, 0) == binding.SD_OK
    assert L.sd_cache_resize(h, t.ref, None) == binding.SD_ERR_ARG
    assert L.sd_cache_copy(h, None, p, 1) == binding.SD_ERR_ARG
    assert L.sd_cache_compact(h, t.ref, None) == binding.SD_OK
    with pytest.raises(ValueError):
        b.cache.fork(t, x[:1], x[:2])
    with pytest.raises(ValueError):
        b.cache.resize(t, x)
    with pytest.raises(ValueError):
        b.cache.resize(t, x[:4].long())
    with pytest.raises(ValueError):
        b.cache.compact(t, x[:2])
    with pytest.raises(ValueError):
        b.cache.compact(binding.PageTables(t.pages, t.length, t.refs[:15].contiguous()))
    with pytest.raises(ValueError):
        binding.PageTables(t.pages, t.length[:3].contiguous(), t.refs)
    assert b.cache.status() == 0


def test_tables_on_another_stream():
    b = Both(6, 6, 40, 8, seed=2)
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)                            # the books are written late, on a stream that is not the cache's
        b.resize([13, 20, 7, 0, 0, 0])
        b.fork([0, 1], [3, 4])
    torch.cuda.synchronize()
    b.same()


@pytest.mark.parametrize("cache_dtype", ["bf16", "e2m1"])
def test_a_prompt_answered_several_times(cache_dtype):
    """A prompt's sequence is forked, the forks and the prompt go on with tokens of their own over pages that resize hands out, some end, the pool is compacted
    on the way: every logit is the one that a cache of the sequence's own gives.  Sequences are run in the same calls on both sides, and the kernels'
    choices go by the call, so that the bits are equal."""
    shape = synth.ModelShape("pages-bf16", 2, 256, 4, 512, 500, 256, "bf16")
    w = synth.make_weights(shape, seed=5)
    n, page, steps, prompt = 5, 16, 24, 37
    dec = binding.Decoder(shape, w, n, 64, 64)
    dec.set_option(binding.SD_OPT_DETERMINISTIC, 1)
    tokens = synth.make_tokens(shape.vocab, 1, prompt, 40)[0]
    forced = torch.randint(0, shape.vocab, (steps, n), generator=torch.Generator().manual_seed(2))
    make = lambda: binding.PagedCache(2, 4, 4, 64, page, 40, n, 256, cache_dtype, stream=dec.stream)  # noqa: E731
    first = i32([0, 1, 2, 3, 4, 5])

    plain = make()                                               # every sequence has read the prompt by itself, in a table of fixed pages
    fixed = torch.arange(n * 6, dtype=torch.int32).view(n, 6).cuda()
    for s in range(n):
        dec.extend(plain, binding.CacheBatch(fixed[s:s + 1].contiguous(), i32([0, prompt]), i32([prompt]), prompt, prompt), tokens)
    want = []
    for t in range(steps):
        batch = binding.CacheBatch(fixed, first, i32([prompt + t + 1] * n), n, 1, 96)
        want.append(dec.extend(plain, batch, forced[t]).cpu())

    cache = make()
    tables = binding.PageTables.empty(cache, n, 6)
    cache.resize(tables, i32([5 * page, 0, 0, 0, 0]))            # a sequence that comes and goes, so that page numbers are not in order
    cache.resize(tables, i32([0, 3 * page, 0, 0, 0]))
    cache.resize(tables, i32([prompt, 3 * page, 0, 0, 0]))
    cache.resize(tables, i32([prompt, 0, 0, 0, 0]))
    dec.extend(cache, binding.CacheBatch(tables.pages[:1], i32([0, prompt]), tables.length[:1], prompt, prompt), tokens)
    cache.fork(tables, i32([0, 0, 0, 0]), i32([1, 2, 3, 4]))
    length = [prompt] * n
    for t in range(steps):
        if t == 9:
            cache.compact(tables)
        length = [l + 1 for l in length]
        cache.resize(tables, i32(length))
        got = dec.extend(cache, binding.CacheBatch(tables.pages, first, tables.length, n, 1, 96), forced[t]).cpu()
        assert torch.equal(got, want[t]), t
    assert cache.status() == 0 and dec.status() == 0
    cache.resize(tables, i32([0] * n))
    assert int(tables.refs.abs().max()) == 0
    for x in (plain, cache, dec):
        x.close()
