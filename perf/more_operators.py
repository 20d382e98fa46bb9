"""Cases that measure the paged cache in 4 bits (append and read back, attention over it), attention whose scores are capped,
biased by distance or masked, and the work on pages: forking, growing, cutting and ending sequences, compacting the pool.

`run` computes them in plain torch operations, or, with `own` set, through the package's binding.  A paged cache is a
pool of pages [n_pages, n_kv_heads, page_len, head_dim] for K and one for V; a table gives each sequence its pages; sequence s
brings the rows first[s] .. first[s+1] of new tokens, the last positions of its len[s].

In 4 bits an element is code * block * scale: a code of e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives, two to a byte, the even
element in the lower half), one e4m3 for every 16 elements of a head, one fp32 for every token and head.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"fp32": 4.0, "bf16": 2.0, "fp16": 2.0, "int8": 1.0, "e4m3": 1.0, "e2m1": 0.5 + 1 / 16}
CODE_MAX = {"int8": 127.0, "e4m3": 448.0, "e2m1": 6.0 * 448.0}

# Sizes: heads, head sizes, batches, prompt and generation lengths are those of the OPT-125M, 1.3B and 6.7B configurations; the
# grouped-query and long-context ones are generic.


def listed():
    return [
        # one user, one token at a time, a short conversation on the smallest model: latency
        dict(name="attend4 one token", op="attend", cache="e2m1", io="bf16", heads=12, kv_heads=12, head_dim=64, page=16, seqs=1, new_lo=1, new_hi=1,
             len_lo=61, len_hi=61, ragged=1),
        # the decode step of a full batch at the 6.7B shape, every sequence at a position of its own
        dict(name="attend4 batch", op="attend", cache="e2m1", io="bf16", heads=32, kv_heads=32, head_dim=128, page=32, seqs=64, new_lo=1, new_hi=1,
             len_lo=1024, len_hi=1536, ragged=2),
        # chunks of prompts, some of them of a few tokens, at the 6.7B shape
        dict(name="attend4 chunks", op="attend", cache="e2m1", io="bf16", heads=32, kv_heads=32, head_dim=128, page=64, seqs=8, new_lo=3, new_hi=1024,
             len_lo=1024, len_hi=4096, ragged=5),
        # one layer's keys and values of a decode step, written and read back
        dict(name="store4 step", op="store", cache="e2m1", io="bf16", heads=12, kv_heads=12, head_dim=64, page=16, seqs=8, new_lo=1, new_hi=1,
             len_lo=129, len_hi=255, ragged=6),
        # the same of a prompt pass, straight out of the fp32 QKV product
        dict(name="store4 prompts", op="store", cache="e2m1", io="fp32", heads=32, kv_heads=32, head_dim=128, page=32, seqs=5, new_lo=700, new_hi=1024,
             len_lo=1024, len_hi=1024, ragged=7),
        # decode over long conversations with a window of the last positions, capped scores, shared key heads
        dict(name="scores window cap", op="scores", cache="bf16", io="bf16", heads=32, kv_heads=8, head_dim=128, page=64, seqs=48, new_lo=1, new_hi=1,
             len_lo=1000, len_hi=12000, ragged=8, cap=50.0, slopes=False, window=2048, documents=0, prefix=False),
        # prompts of many documents packed one behind the other: a token sees its own document, a few tokens (separators) nothing
        dict(name="scores documents cap", op="scores", cache="bf16", io="bf16", heads=32, kv_heads=32, head_dim=64, page=32, seqs=2, new_lo=3900, new_hi=4096,
             len_lo=4096, len_hi=4096, ragged=9, cap=30.0, slopes=False, window=0, documents=450, prefix=False),
        # prompts whose first part is seen by all of its tokens, scores biased by distance, over an 8-bit cache
        dict(name="scores prefix slopes", op="scores", cache="int8", io="bf16", heads=12, kv_heads=12, head_dim=64, page=16, seqs=9, new_lo=500, new_hi=1001,
             len_lo=500, len_hi=1500, ragged=10, cap=0.0, slopes=True, window=0, documents=0, prefix=True),
        # one request answered four times: its sequence is forked and the forks grow, 125M shape
        dict(name="branch one", op="branch", kv_heads=12, head_dim=64, page=16, layers=2, live=1, ways=3, len_lo=61, len_hi=61, grow=1, ragged=11),
        # a batch of requests answered three times each: prompts are forked, some answers end, some are cut back, the others grow
        dict(name="branch batch", op="branch", kv_heads=32, head_dim=128, page=32, layers=4, live=48, ways=2, len_lo=33, len_hi=190, grow=40, ragged=12),
        # a small pool after some requests have ended
        dict(name="compact small", op="compact", kv_heads=12, head_dim=64, page=16, layers=2, seqs=5, len_lo=20, len_hi=129, spare=1.0, ragged=13),
        # a large one, half empty, pages of sequences shared between forks
        dict(name="compact large", op="compact", kv_heads=32, head_dim=128, page=32, layers=4, seqs=40, len_lo=64, len_hi=512, spare=1.0, ragged=14),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "store", "scores", "scores", "scores", "branch", "compact"])
    if op in ("branch", "compact"):
        head_dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64])
        kv_heads, layers = rng.choice([1, 5, 8, 12, 32]), rng.randint(1, 4)
        seqs = _log_int(rng, 1, 40)
        pages = int(1.2e9 / (4 * layers * kv_heads * page * head_dim)) // (4 * seqs) - 3     # of a sequence, with its forks, in 1.2 GB
        len_hi = _log_int(rng, 1, max(page, min(2000, pages * page)))
        case = dict(op=op, kv_heads=kv_heads, head_dim=head_dim, page=page, layers=layers, len_lo=rng.randint(1, len_hi), len_hi=len_hi, ragged=rng.randrange(1 << 30))
        if op == "branch":
            return dict(case, live=seqs, ways=rng.randint(1, 3), grow=_log_int(rng, 1, 64))
        return dict(case, seqs=seqs, spare=round(rng.uniform(0.1, 1.5), 2))
    head_dim = rng.choice([64, 128])
    kv_heads, group = rng.choice([(12, 1), (32, 1), (8, 4), (5, 1), (4, 7), (1, 8)])
    case = dict(op=op, cache="e2m1", io=rng.choice(["bf16", "bf16", "fp32"]), heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim,
                page=rng.choice([16, 32, 64]), ragged=rng.randrange(1 << 30))
    if op == "store":
        seqs = _log_int(rng, 1, 48)
        new_hi = min(4096, _log_int(rng, 1, max(1, 4096 * 32 // (seqs * kv_heads))))
        more = rng.randint(0, 300)
        return dict(case, seqs=seqs, new_lo=rng.randint(1, new_hi), new_hi=new_hi, len_lo=new_hi + more, len_hi=new_hi + more)
    seqs = _log_int(rng, 1, 64)
    len_hi = _log_int(rng, 40, min(65536, 98304 * 32 // (seqs * kv_heads)))
    new_hi = 1 if rng.random() < 0.5 else min(len_hi, _log_int(rng, 2, 1024))
    # never more work than the largest listed case: 8 chunks of up to 1024 queries over up to 4096 positions of 32 heads
    while new_hi > 1 and seqs * new_hi * len_hi * case["heads"] > 4 * 1024 * 2500 * 32:
        new_hi = max(1, new_hi // 2)
    case.update(seqs=seqs, new_lo=rng.choice([1, new_hi]), new_hi=new_hi, len_lo=rng.randint(max(new_hi, len_hi // 4), len_hi), len_hi=len_hi)
    if op == "scores":
        kind = rng.randrange(4)                              # a window, documents, a prefix, no mask
        case.update(cache=rng.choice(["bf16", "bf16", "int8", "e4m3", "e2m1"]), cap=rng.choice([0.0, 15.0, 30.0, 50.0]), slopes=rng.random() < 0.5,
                    window=_log_int(rng, 16, 4096) if kind == 0 else 0, documents=_log_int(rng, 20, 2000) if kind == 1 else 0, prefix=kind == 2)
        if kind == 3 and not case["slopes"] and case["cap"] == 0:
            case["cap"] = 30.0
    return case


# ---- what belongs to the case and not to the seed -----------------------------------------------

def _lengths(case):
    """New tokens and positions of each sequence."""
    r = random.Random(case["ragged"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    return new, [max(n, r.randint(case["len_lo"], case["len_hi"])) for n in new]


def _ranges(case):
    """For each sequence its new tokens' first and last visible position, as lists."""
    new, length = _lengths(case)
    r = random.Random(case["ragged"] + 1)
    out = []
    for n, l in zip(new, length):
        pos = range(l - n, l)
        lo, hi = [0] * n, list(pos)
        if case["window"]:
            lo = [max(0, p - case["window"] + 1) for p in pos]
        if case["documents"]:                                # borders anywhere in the sequence
            start, starts = 0, []
            end = r.randint(1, 2 * case["documents"])
            for p in range(l):
                if p == end:
                    start, end = p, p + r.randint(1, 2 * case["documents"])
                starts.append(start)
            lo = [starts[p] for p in pos]
            for i in range(0, n, 211):                       # separators see nothing
                lo[i] = hi[i] + 1
        if case["prefix"]:
            prefix = r.randint(0, l)
            hi = [max(p, prefix - 1) for p in pos]
        out.append((lo, hi))
    return out


def _branches(case):
    """Lengths of the live sequences, and the length that each row of the table is to have after the fork."""
    r = random.Random(case["ragged"])
    length = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["live"])]
    after = length + [l for l in length for _ in range(case["ways"])]
    target = []
    for i, l in enumerate(after):
        what = r.random() if len(after) > 8 else 1.0
        target.append(0 if what < 0.1 else r.randint(0, l) if what < 0.25 else l + r.randint(1, case["grow"]))
    return length, target


def _counts(case):
    """Lengths of a pool's sequences; every third one shares its whole pages with the one before it."""
    r = random.Random(case["ragged"])
    length = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]
    for s in range(2, case["seqs"], 3):
        length[s] = length[s - 1]
    used = sum((1 if l % case["page"] else 0) if s >= 2 and s % 3 == 2 else -(-l // case["page"]) for s, l in enumerate(length))
    return length, used, used + max(2, int(used * case["spare"]))


def work(case):
    op = case["op"]
    if op in ("branch", "compact"):
        page_bytes = 2 * case["layers"] * case["kv_heads"] * case["page"] * case["head_dim"] * 2
        if op == "branch":
            length, target = _branches(case)
            copies = case["ways"] * sum(1 for l in length if l % case["page"])
            tables = sum(-(-t // case["page"]) for t in target) * 8
        else:
            length, used, n_pages = _counts(case)
            copies = used * (n_pages - used) // n_pages      # on average: the used pages lie anywhere
            tables = sum(-(-l // case["page"]) for l in length) * 8 + n_pages * 8
        return {"bytes": 2 * copies * page_bytes + tables, "flops": 0}
    new, length = _lengths(case)
    H, K, d, io = case["heads"], case["kv_heads"], case["head_dim"], BYTES[case["io"]]
    per_token = 2 * K * (d * BYTES[case["cache"]] + (4 if case["cache"] in CODE_MAX else 0))
    if op == "store":                                        # read and written in 4 bits, then read from there and written out
        return {"bytes": 2 * (sum(new) * 2 * K * d * io + sum(new) * per_token), "flops": 4 * sum(new) * K * d}
    if op == "attend":
        seen, keys = sum(n * l - n * (n - 1) // 2 for n, l in zip(new, length)), sum(length)
    else:
        seen = keys = 0
        for lo, hi in _ranges(case):
            some = [(a, b) for a, b in zip(lo, hi) if a <= b]
            seen += sum(b - a + 1 for a, b in some)
            keys += max(b for _, b in some) + 1 - min(a for a, _ in some) if some else 0
    return {"bytes": keys * per_token + 2 * sum(new) * H * d * io, "flops": 4 * seen * H * d}


# ---- inputs --------------------------------------------------------------------------------------

def _round_e4m3(y):
    """To the nearest number m * 2^e with 4 bits of m in [0.5, 1) and e at least -5, ties to even, at most 448."""
    _, e = torch.frexp(y)
    e = e.clamp_min(-5) - 4
    return torch.ldexp(torch.round(torch.ldexp(y, -e)), e).clamp(-448.0, 448.0)


def _quantise(x, kind):
    """The parts of rows along the last axis: codes, (blocks,) scales.  The scale is the row's largest magnitude over the largest
    value of a code (and block), held in 32 bits; what is rounded is the nearest, ties to even, decided in 64 bits."""
    top = torch.tensor(CODE_MAX[kind], device=x.device)      # a tensor, so that the division is a division
    scale = x.abs().amax(-1) / top
    safe = torch.where(scale > 0, scale, torch.ones_like(scale)).double().unsqueeze(-1)
    if kind == "e2m1":
        y = x.double().unflatten(-1, (-1, 16))
        block = _round_e4m3(y.abs().amax(-1) / (6.0 * safe))
        block = torch.where((scale > 0).unsqueeze(-1), block, torch.zeros_like(block))
        unit = block.unsqueeze(-1) * safe.unsqueeze(-1)
        a = (y / torch.where(unit > 0, unit, torch.ones_like(unit))).abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        a = torch.where(unit > 0, (torch.round(a / step) * step).clamp_max(6.0), torch.zeros_like(a))
        code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | ((y < 0).to(torch.uint8) << 3)
        code = code.flatten(-2)
        return code[..., 0::2] | (code[..., 1::2] << 4), block.to(torch.float8_e4m3fn), scale
    y = x.double() / safe
    y = torch.round(y) if kind == "int8" else _round_e4m3(y)
    y = torch.where((scale > 0).unsqueeze(-1), y.clamp(-CODE_MAX[kind], CODE_MAX[kind]), torch.zeros_like(y))
    return y.to(TYPES[kind]), scale


def _parts(kind, name):
    """Names of the pools that hold K or V."""
    return [name] + [name + "_block"] * (kind == "e2m1") + [name + "_scale"] * (kind in CODE_MAX)


def _pools(kind, n_pages, kv_heads, page, head_dim):
    shape = (n_pages, kv_heads, page)
    out = {}
    for n in ("k", "v"):
        out[n] = torch.zeros(shape + ((head_dim // 2,) if kind == "e2m1" else (head_dim,)), dtype=torch.uint8 if kind == "e2m1" else TYPES[kind], device=DEVICE)
        if kind == "e2m1":
            out[n + "_block"] = torch.zeros(shape + (head_dim // 16,), dtype=torch.float8_e4m3fn, device=DEVICE)
        if kind in CODE_MAX:
            out[n + "_scale"] = torch.zeros(shape, dtype=torch.float32, device=DEVICE)
    return out


def _bytes_of(t):
    return t.view(torch.uint8) if t.dtype in (torch.float8_e4m3fn, torch.int8) else t


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    if case["op"] in ("branch", "compact"):
        return _prepare_pages(case, g)
    new, length = _lengths(case)
    K, d, page, kind = case["kv_heads"], case["head_dim"], case["page"], case["cache"]
    n_tok = sum(new)
    per_seq = (max(length) + page - 1) // page
    used = [(l + page - 1) // page for l in length]
    n_pages = sum(used) + 3
    perm = torch.randperm(n_pages, device=DEVICE, generator=g)
    pages = torch.full((len(new), per_seq), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for s, u in enumerate(used):
        pages[s, :u] = perm[at:at + u].to(torch.int32)
        at += u
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    first = torch.tensor(starts, dtype=torch.int32, device=DEVICE)
    lens = torch.tensor(length, dtype=torch.int32, device=DEVICE)
    st = dict(case=case, pages=pages, first=first, len=lens, n_tokens=n_tok, max_new=max(new), max_len=max(length))
    if case["op"] == "scores":
        ranges = _ranges(case)
        st["lo"] = torch.tensor([a for lo, _ in ranges for a in lo], dtype=torch.int32, device=DEVICE)
        st["hi"] = torch.tensor([b for _, hi in ranges for b in hi], dtype=torch.int32, device=DEVICE)
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["heads"] + 1, device=DEVICE) / case["heads"]) if case["slopes"] else None
    if own:
        from paper_2307_02628_b200 import binding
        st["cache"] = binding.PagedCache(1, case["heads"], K, d, page, n_pages, max_seqs=len(new), max_tokens=n_tok, dtype=kind,
                                         stream=torch.cuda.current_stream())
        st["batch"] = binding.CacheBatch(pages, first, lens, n_tokens=n_tok, max_new=max(new), max_len=max(length))
        if case["op"] == "scores":
            st["scores"] = binding.Scores(cap=case["cap"], slopes=st["slopes"], window=case["window"],
                                          lo=st["lo"] if case["documents"] else None, hi=st["hi"] if case["prefix"] else None)
        pool = st["cache"].layer(0)
    else:
        pool = _pools(kind, n_pages, K, page, d)
    # keys have channels of different sizes, a few of them large, as trained models' keys do; values are even
    gain = torch.exp(0.3 * torch.randn(K, 1, d, device=DEVICE, generator=g))
    gain[:, :, :2] *= 3.0
    if case["op"] != "store":
        for n in ("k", "v"):
            for lo in range(0, n_pages, 4096):
                hi = min(n_pages, lo + 4096)
                x = torch.randn(hi - lo, K, page, d, device=DEVICE, generator=g)
                if n == "k":
                    x *= gain
                if kind in CODE_MAX:
                    for name, part in zip(_parts(kind, n), _quantise(x, kind)):
                        _bytes_of(pool[name])[lo:hi].copy_(_bytes_of(part))
                else:
                    pool[n][lo:hi].copy_(x)
    st["pool"] = pool
    if case["op"] == "store":
        # rows of a QKV product: keys and values are slices of wider rows
        qkv = torch.randn(n_tok, (case["heads"] + 2 * K) * d, device=DEVICE, generator=g)
        qkv[:, case["heads"] * d:(case["heads"] + K) * d] *= gain.reshape(-1)
        qkv = qkv.to(TYPES[case["io"]])
        st["k"] = qkv[:, case["heads"] * d:(case["heads"] + K) * d].unflatten(1, (K, d))
        st["v"] = qkv[:, (case["heads"] + K) * d:].unflatten(1, (K, d))
    else:
        # scores reach some tens where they are capped, as they do where models need it
        q = torch.randn(n_tok, case["heads"], d, device=DEVICE, generator=g) * (4.0 if case.get("cap") else 1.0)
        st["q"] = q.to(TYPES[case["io"]])
    return st


def _prepare_pages(case, g):
    """Pools of a cache in bf16, and the books: a table, lengths, and how many sequences hold each page, in one tensor, so that a
    pass can begin with them as they were."""
    page, layers = case["page"], case["layers"]
    if case["op"] == "branch":
        length, target = _branches(case)
        rows, columns = len(target), max(1, -(-max(target + length) // page)) + 1
        n_pages = sum(-(-l // page) for l in length) + sum(-(-max(t, 1) // page) + 2 for t in target) + 3
        held = [-(-l // page) for l in length] + [0] * (rows - len(length))
        share = [False] * rows
    else:
        length, _, n_pages = _counts(case)
        rows, columns = len(length), -(-max(length) // page) + 1
        held = [-(-l // page) for l in length]
        share = [s >= 2 and s % 3 == 2 for s in range(rows)]
    perm = torch.randperm(n_pages, device=DEVICE, generator=g).to(torch.int32)
    books = torch.zeros(rows * columns + rows + n_pages, dtype=torch.int32, device=DEVICE)
    pages, lens, refs = books[:rows * columns].view(rows, columns), books[rows * columns:rows * (columns + 1)], books[rows * (columns + 1):]
    pages.fill_(-1)
    lens[:len(length)] = torch.tensor(length, dtype=torch.int32, device=DEVICE)
    at = 0
    for s, n in enumerate(held):
        own_from = length[s] // page if share[s] else 0
        if share[s]:
            pages[s, :own_from] = pages[s - 1, :own_from]
        pages[s, own_from:n] = perm[at:at + n - own_from]
        at += n - own_from
    entries = pages.flatten().long()
    refs.index_add_(0, entries.clamp_min(0), (entries >= 0).to(torch.int32))
    st = dict(case=case, books=books, start=books.clone(), pages=pages, len=lens, refs=refs)
    if case["op"] == "branch":
        live, ways = case["live"], case["ways"]
        st["src"] = torch.arange(live, device=DEVICE, dtype=torch.int32).repeat_interleave(ways)
        st["dst"] = torch.arange(live, live * (1 + ways), device=DEVICE, dtype=torch.int32)
        st["target"] = torch.tensor(target, dtype=torch.int32, device=DEVICE)
    else:
        st["used"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    if own:
        from paper_2307_02628_b200 import binding
        st["cache"] = binding.PagedCache(layers, case["kv_heads"], case["kv_heads"], case["head_dim"], page, n_pages, max_seqs=rows, max_tokens=1,
                                         dtype="bf16", stream=torch.cuda.current_stream())
        st["tables"] = binding.PageTables(pages, lens, refs)
        st["pools"] = [st["cache"].layer(i)[n] for i in range(layers) for n in ("k", "v")]
    else:
        st["pools"] = [t for _ in range(layers) for t in _pools("bf16", n_pages, case["kv_heads"], page, case["head_dim"]).values()]
    for t in st["pools"]:
        t.normal_(generator=g)
    return st


# ---- plain forms ---------------------------------------------------------------------------------

def _rows(st):
    """Sequence and position of every new token."""
    first = st["first"].long()
    count = first[1:] - first[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEVICE), count, output_size=st["n_tokens"])
    pos = st["len"].long()[seq] - count[seq] + torch.arange(st["n_tokens"], device=DEVICE) - first[seq]
    return seq, pos


def _slots(st, seq, pos):
    page = st["case"]["page"]
    return st["pages"].long()[seq, pos // page], pos % page


def _values(st, name, page, slot):
    """Entries of the pool as 32-bit values [..., kv_heads, head_dim]."""
    kind, pool = st["case"]["cache"], st["pool"]
    x = pool[name][page, :, slot]
    if kind == "e2m1":
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEVICE)
        x = table[torch.stack((x & 15, x >> 4), -1).flatten(-2).int()]
        x = (x.unflatten(-1, (-1, 16)) * pool[name + "_block"][page, :, slot].float().unsqueeze(-1)).flatten(-2)
    x = x.float()
    return x * pool[name + "_scale"][page, :, slot].unsqueeze(-1) if kind in CODE_MAX else x


def _store(st):
    seq, pos = _rows(st)
    page, slot = _slots(st, seq, pos)
    for n in ("k", "v"):
        for name, part in zip(_parts("e2m1", n), _quantise(st[n].float(), "e2m1")):
            _bytes_of(st["pool"][name])[page, :, slot] = _bytes_of(part)
    return {n: _values(st, n, page, slot).to(TYPES[st["case"]["io"]]) for n in ("k", "v")}


def _attend(st):
    case = st["case"]
    H, K, d = case["heads"], case["kv_heads"], case["head_dim"]
    seqs, top, most = case["seqs"], st["max_len"], st["max_new"]
    every = torch.arange(top, device=DEVICE)
    page, slot = _slots(st, torch.arange(seqs, device=DEVICE).unsqueeze(1), every.unsqueeze(0))
    page = page.clamp_min(0)                                             # past a sequence's end: masked below
    seq, pos = _rows(st)
    at = pos - (st["len"].long() - (st["first"][1:] - st["first"][:-1]).long())[seq]

    def spread(rows, fill):                                              # [n_tokens] -> [seqs, most]
        out = torch.full((seqs, most), fill, device=DEVICE, dtype=torch.long)
        out[seq, at] = rows.long()
        return out

    q = torch.zeros(seqs, most, H, d, device=DEVICE)
    q[seq, at] = st["q"].float()
    q = q.unflatten(2, (K, H // K)).permute(0, 2, 3, 1, 4).flatten(2, 3)     # [seqs, K, group * most, d]
    k = _values(st, "k", page, slot).transpose(1, 2)                         # [seqs, K, top, d]
    s = (q @ k.transpose(2, 3) * d ** -0.5).unflatten(2, (H // K, most))     # [seqs, K, group, most, top]
    del k
    dead = every > spread(st["hi"] if case["op"] == "scores" else pos, -1).unsqueeze(-1)
    if case["op"] == "scores":
        if case["cap"]:
            s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
        dead |= every < spread(st["lo"], 0).unsqueeze(-1)
        if case["slopes"]:
            away = (every - spread(pos, 0).unsqueeze(-1)).abs().float()          # [seqs, most, top]
            s -= st["slopes"].unflatten(0, (K, H // K))[None, :, :, None, None] * away[:, None, None]
            del away
    s.masked_fill_(dead[:, None, None], float("-inf"))
    del dead
    s -= s.amax(-1, keepdim=True).clamp_min(-3e38)                           # a row without keys has no maximum
    s.exp_()
    total = s.sum(-1, keepdim=True)
    o = s.flatten(2, 3) @ _values(st, "v", page, slot).transpose(1, 2)
    o = o.unflatten(2, (H // K, most)) / torch.where(total > 0, total, 1.0)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, at].to(TYPES[case["io"]])


def _free(refs):
    """Pages that nobody holds, in order, and behind them the others."""
    return torch.argsort((refs != 0).to(torch.uint8), stable=True)


def _move(st, source, target):
    for t in st["pools"]:
        t.index_copy_(0, target, t.index_select(0, source))


def _branch(st):
    """Forks share whole pages and get a copy of the last one where it is not full; then every row takes its new length: pages past it
    are given back, a page that is kept in part and held by others too is copied, missing pages are added.  New pages are
    the lowest free ones, row by row, a copy before the missing ones."""
    case, page = st["case"], st["case"]["page"]
    st["books"].copy_(st["start"])
    pages, lens, refs = st["pages"], st["len"], st["refs"]
    column = torch.arange(pages.shape[1], device=DEVICE)
    src, dst = st["src"].long(), st["dst"].long()
    length, rows = lens[src].long(), pages[src].long()
    whole, last = column < (length // page).unsqueeze(1), (length // page).unsqueeze(1)
    part = length % page > 0
    old = rows.gather(1, last).squeeze(1).clamp_min(0)
    new = torch.where(part, _free(refs)[part.long().cumsum(0) - 1], old)
    _move(st, old[part], new[part])
    refs.index_add_(0, rows.clamp_min(0).flatten(), whole.to(torch.int32).flatten())
    refs.index_add_(0, new, part.to(torch.int32))
    fork = torch.where(whole, rows, -1).scatter(1, last, torch.where(part, new, -1).unsqueeze(1))
    pages[dst], lens[dst] = fork.to(torch.int32), length.to(torch.int32)

    length, target, rows = lens.long(), st["target"].long(), pages.long()
    have, want = (length + page - 1) // page, (target + page - 1) // page
    given = (column >= want.unsqueeze(1)) & (column < have.unsqueeze(1))
    refs.index_add_(0, rows.clamp_min(0).flatten(), -given.to(torch.int32).flatten())
    kept = torch.minimum(length, target)
    last = (kept // page).unsqueeze(1)
    old = rows.gather(1, last).squeeze(1).clamp_min(0)
    copied = (kept % page > 0) & (refs[old] > 1)
    more = (want - have).clamp_min(0)
    begin = (copied + more).cumsum(0) - (copied + more)
    free = _free(refs)
    new = torch.where(copied, free[begin.clamp_max(free.numel() - 1)], old)
    _move(st, old[copied], new[copied])
    refs.index_add_(0, old, -copied.to(torch.int32))
    refs.index_add_(0, new, copied.to(torch.int32))
    rows = torch.where(given, -1, rows)
    rows.scatter_(1, last, torch.where(copied, new, rows.gather(1, last).squeeze(1)).unsqueeze(1))
    added = (column >= have.unsqueeze(1)) & (column < want.unsqueeze(1))
    order = (begin + copied).unsqueeze(1) + (column - have.unsqueeze(1)).clamp_min(0)
    which = free[order.clamp_max(free.numel() - 1)]
    refs.index_add_(0, which.flatten(), added.to(torch.int32).flatten())
    pages.copy_(torch.where(added, which, rows))
    lens.copy_(target)
    return [pages, lens, refs] + st["pools"]


def _compact(st):
    """The used pages from number `used` on move, in order, to the free ones below it, in order."""
    st["books"].copy_(st["start"])
    pages, refs = st["pages"], st["refs"]
    number = torch.arange(refs.numel(), device=DEVICE)
    held = refs > 0
    used = held.sum()
    source, target = number[held & (number >= used)], number[~held & (number < used)]
    _move(st, source, target)
    place = number.scatter(0, source, target)
    columns = torch.arange(pages.shape[1], device=DEVICE)
    inside = columns < ((st["len"].long() + st["case"]["page"] - 1) // st["case"]["page"]).unsqueeze(1)
    pages.copy_(torch.where(inside, place[pages.long().clamp_min(0)], pages.long()))
    refs.copy_(torch.zeros_like(refs).index_add_(0, place, refs))
    st["used"].copy_(used)
    return [pages, st["len"], refs, st["used"]] + st["pools"]


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"attend": _attend, "scores": _attend, "store": _store, "branch": _branch, "compact": _compact}[op](st)
    cache = st["cache"]
    if op == "attend":
        return cache.attention(0, st["q"], st["batch"])
    if op == "scores":
        return cache.attention(0, st["q"], st["batch"], scores=st["scores"])
    if op == "store":
        cache.append(0, st["k"], st["v"], st["batch"])
        k, v = cache.read(0, st["batch"], TYPES[st["case"]["io"]])
        return {"k": k, "v": v}
    st["books"].copy_(st["start"])
    if op == "branch":
        cache.fork(st["tables"], st["src"], st["dst"])
        cache.resize(st["tables"], st["target"])
        return [st["pages"], st["len"], st["refs"]] + st["pools"]
    cache.compact(st["tables"], st["used"])
    return [st["pages"], st["len"], st["refs"], st["used"]] + st["pools"]


# ---- the definitions in 64 bits --------------------------------------------------------------------

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(y, values):
    """The nearest of the increasing values to each y >= 0; between two, halfway, the one with an even index."""
    v = torch.tensor(values, dtype=torch.float64, device=y.device)
    at = torch.searchsorted(v, y).clamp(1, len(values) - 1)
    below, above = y - v[at - 1], v[at] - y
    up = (below > above) | ((below == above) & (at % 2 == 0))
    return v[torch.where(up, at, at - 1)]


def _stored(x):
    """What the 4-bit cache gives back for rows x, in 64 bits."""
    x = x.double()
    scale = (x.abs().amax(-1, keepdim=True).float() / torch.tensor(2688.0, device=x.device)).double()        # the cache holds it in 32 bits
    e4m3 = [m * 2.0 ** -9 for m in range(8)] + [m * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8, 16)][:-1]       # at most 448
    out = []
    for lo in range(0, x.shape[-1], 16):
        part = x[..., lo:lo + 16]
        block = torch.where(scale > 0, _nearest(part.abs().amax(-1, keepdim=True) / (6 * scale), e4m3), 0.0)
        unit = block * scale
        out.append(torch.where(unit > 0, torch.sign(part) * _nearest(part.abs() / unit, _E2M1) * unit, 0.0))
    return torch.cat(out, -1)


def exact(case, seed):
    if case["op"] in ("branch", "compact"):
        return None                                          # whole numbers, and pages as they were
    st = prepare(case, seed)
    if case["op"] == "store":
        return {n: _stored(st[n]) for n in ("k", "v")}
    new, length = _lengths(case)
    K, d, page, kind = case["kv_heads"], case["head_dim"], case["page"], case["cache"]

    def sequence(name, s):
        ids = st["pages"][s, :(length[s] + page - 1) // page].long()
        x = st["pool"][name][ids]                             # [pages, K, page, ...]
        if kind == "e2m1":
            code = torch.stack((x % 16, x // 16), -1).flatten(-2).long()
            x = torch.tensor(_E2M1, dtype=torch.float64, device=DEVICE)[code % 8] * (1 - 2 * (code // 8)).double()
            x = x * st["pool"][name + "_block"][ids].double().repeat_interleave(16, -1)
        x = x.double()
        if kind in CODE_MAX:
            x = x * st["pool"][name + "_scale"][ids].double().unsqueeze(-1)
        return x.transpose(0, 1).reshape(K, -1, d)[:, :length[s]]

    scores = case["op"] == "scores"
    ranges = _ranges(case) if scores else [([0] * n, list(range(l - n, l))) for n, l in zip(new, length)]
    outs = []
    row = 0
    group = case["heads"] // K
    for s, (n, l) in enumerate(zip(new, length)):
        k, v = sequence("k", s), sequence("v", s)
        key = torch.arange(l, device=DEVICE)
        for lo in range(0, n, 256):
            hi = min(n, lo + 256)
            q = st["q"][row + lo:row + hi].double().reshape(hi - lo, K, group, d)
            p = torch.einsum("nkgd,kjd->kgnj", q, k) / math.sqrt(d)
            if scores and case["cap"]:
                p = case["cap"] * torch.tanh(p / case["cap"])
            if scores and case["slopes"]:
                at = torch.arange(l - n + lo, l - n + hi, device=DEVICE).unsqueeze(1)
                p = p - st["slopes"].double().reshape(K, group, 1, 1) * (key - at).abs()
            first, last = (torch.tensor(r[lo:hi], device=DEVICE).unsqueeze(1) for r in ranges[s])
            hidden = (key < first) | (key > last)
            p = torch.softmax(p.masked_fill(hidden, float("-inf")), dim=-1)
            p = torch.where(hidden.all(1, keepdim=True), 0.0, p)
            outs.append(torch.einsum("kgnj,kjd->nkgd", p, v).reshape(hi - lo, case["heads"], d))
        row += n
    return torch.cat(outs)
