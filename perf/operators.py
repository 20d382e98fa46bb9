"""Cases that measure the serving operators: the paged 8-bit cache (append, read back), attention of new tokens
over it, and token selection with each row's own settings.

`run` computes them in plain torch operations, or, with `own` set, through the package's binding.  A paged cache is a
pool of pages [n_pages, n_kv_heads, page_len, head_dim] for K and one for V, with one fp32 scale per token and head
where it is held in 8 bits; a table gives each sequence its pages; sequence s brings the rows first[s] .. first[s+1]
of new tokens, the last positions of its len[s].
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "int8": 1, "e4m3": 1}
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}

# Sizes: heads, head sizes, batches, prompt and generation lengths and the vocabulary are those of the OPT-125M, 1.3B and
# 6.7B configurations; the grouped-query and long-context ones are generic.


def listed():
    return [
        # one user, one token at a time, a short conversation on the smallest model: latency
        dict(name="attend one token", op="attend", cache="bf16", io="bf16", heads=12, kv_heads=12, head_dim=64, page=16, seqs=1, new_lo=1, new_hi=1,
             len_lo=61, len_hi=61, ragged=1),
        # the decode step of a full batch at the 6.7B shape: every sequence at a position of its own
        dict(name="attend batch int8", op="attend", cache="int8", io="bf16", heads=32, kv_heads=32, head_dim=128, page=32, seqs=64, new_lo=1, new_hi=1,
             len_lo=1024, len_hi=1536, ragged=2),
        # few users with long documents, shared key heads: the length has to be split
        dict(name="attend long gqa", op="attend", cache="bf16", io="bf16", heads=32, kv_heads=8, head_dim=128, page=64, seqs=3, new_lo=1, new_hi=1,
             len_lo=20000, len_hi=65521, ragged=3),
        # a serving step that mixes single tokens with prompt chunks, 1.3B shape
        dict(name="attend mixed e4m3", op="attend", cache="e4m3", io="bf16", heads=32, kv_heads=32, head_dim=64, page=16, seqs=33, new_lo=1, new_hi=331,
             len_lo=350, len_hi=1500, ragged=4),
        # chunks of long prompts at the 6.7B shape
        dict(name="attend chunks bf16", op="attend", cache="bf16", io="bf16", heads=32, kv_heads=32, head_dim=128, page=64, seqs=8, new_lo=1000, new_hi=1024,
             len_lo=1024, len_hi=4096, ragged=5),
        # one layer's keys and values of a decode step, written and read back
        dict(name="store step int8", op="store", cache="int8", io="bf16", heads=12, kv_heads=12, head_dim=64, page=16, seqs=8, new_lo=1, new_hi=1,
             len_lo=129, len_hi=255, ragged=6),
        # the same of a prompt pass, straight out of the fp32 QKV product
        dict(name="store prompts e4m3", op="store", cache="e4m3", io="fp32", heads=32, kv_heads=32, head_dim=128, page=32, seqs=5, new_lo=700, new_hi=1024,
             len_lo=1024, len_hi=1024, ragged=7),
        # a short sequence leaves the cache (to be moved or shared)
        dict(name="load one e4m3", op="load", cache="e4m3", io="bf16", heads=32, kv_heads=32, head_dim=64, page=16, seqs=1, new_lo=512, new_hi=512,
             len_lo=512, len_hi=512, ragged=8),
        # a whole batch does
        dict(name="load batch int8", op="load", cache="int8", io="bf16", heads=32, kv_heads=32, head_dim=128, page=32, seqs=24, new_lo=900, new_hi=1500,
             len_lo=900, len_hi=1500, ragged=9),
        # token selection: one user; a small vocabulary; a full batch
        dict(name="sample one", op="sample", rows=1, vocab=50272, spread=1.5),
        dict(name="sample small vocabulary", op="sample", rows=33, vocab=1021, spread=1.0),
        dict(name="sample batch", op="sample", rows=256, vocab=50272, spread=2.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "load", "sample"])
    if op == "sample":
        return dict(op=op, rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 500, 50272), spread=round(rng.uniform(0.3, 3.0), 2))
    head_dim = rng.choice([64, 128])
    kv_heads, group = rng.choice([(12, 1), (32, 1), (8, 4), (5, 1), (4, 7), (1, 8)])
    case = dict(op=op, cache=rng.choice(["bf16", "int8", "e4m3"]), io=rng.choice(["bf16", "bf16", "fp32"]), heads=kv_heads * group, kv_heads=kv_heads,
                head_dim=head_dim, page=rng.choice([16, 32, 64]), ragged=rng.randrange(1 << 30))
    if op == "attend":
        seqs = _log_int(rng, 1, 64)
        len_hi = _log_int(rng, 40, min(65536, 98304 * 32 // (seqs * kv_heads)))
        new_hi = 1 if rng.random() < 0.5 else min(len_hi, _log_int(rng, 2, 1024))
        # never more work than the largest listed case: 8 x 1024 queries over 4096 positions of 32 heads
        while new_hi > 1 and seqs * new_hi * len_hi * case["heads"] > 8 * 1024 * 4096 * 16:
            new_hi = max(1, new_hi // 2)
        case.update(seqs=seqs, new_lo=rng.choice([1, new_hi]), new_hi=new_hi, len_lo=rng.randint(max(new_hi, len_hi // 4), len_hi), len_hi=len_hi)
    else:
        seqs = _log_int(rng, 1, 48)
        new_hi = _log_int(rng, 1, max(1, 24 * 1024 * 32 // (seqs * kv_heads * 2)))
        new_hi = min(new_hi, 4096)
        new_lo = rng.randint(1, new_hi)
        more = 0 if op == "load" else rng.randint(0, 300)
        case.update(seqs=seqs, new_lo=new_lo, new_hi=new_hi, len_lo=new_hi + more, len_hi=new_hi + more)
    return case


def _lengths(case):
    """New tokens and positions of each sequence: they belong to the case, not to the seed."""
    r = random.Random(case["ragged"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    length = [max(n, r.randint(case["len_lo"], case["len_hi"])) for n in new]
    if case["op"] == "load":                 # whole sequences are read
        length = list(new)
    return new, length


def work(case):
    if case["op"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * 4 + 24), "flops": 4 * case["rows"] * case["vocab"]}
    new, length = _lengths(case)
    H, K, d, io = case["heads"], case["kv_heads"], case["head_dim"], BYTES[case["io"]]
    per_token = 2 * K * (d * BYTES[case["cache"]] + (4 if case["cache"] in CODE_MAX else 0))
    if case["op"] == "attend":
        seen = sum(n * l - n * (n - 1) // 2 for n, l in zip(new, length))
        return {"bytes": sum(length) * per_token + 2 * sum(new) * H * d * io, "flops": 4 * seen * H * d}
    plain = sum(new) * 2 * K * d * io
    # stored: the tokens are read and written in the cache's type, then read from it and written out
    return {"bytes": plain + sum(new) * per_token if case["op"] == "load" else 2 * (plain + sum(new) * per_token), "flops": 4 * sum(new) * K * d}


def _quantise(x, kind):
    """Codes and scales of rows along the last axis.  The scale is the row's largest magnitude over the largest code, held in
    32 bits; a code is the nearest to x / scale, ties to even, decided in 64 bits (a quotient rounded to 32 first can land on
    a tie).  A row of zeros has scale 0 and codes 0."""
    top = torch.tensor(CODE_MAX[kind], device=x.device)      # a tensor, so that the division is a division
    scale = x.abs().amax(-1) / top
    y = x.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double().unsqueeze(-1)
    if kind == "int8":
        y = torch.round(y)
    else:                                                    # a number m * 2^e, m in [0.5, 1): m keeps 4 bits, e is at least -5
        _, e = torch.frexp(y)
        e = e.clamp_min(-5) - 4
        y = torch.ldexp(torch.round(torch.ldexp(y, -e)), e)
    y = torch.where((scale > 0).unsqueeze(-1), y.clamp(-CODE_MAX[kind], CODE_MAX[kind]), torch.zeros_like(y))
    return y.to(TYPES[kind]), scale


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, g)
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
    if own:
        from paper_2307_02628_b200 import binding
        st["cache"] = binding.PagedCache(1, case["heads"], K, d, page, n_pages, max_seqs=len(new), max_tokens=n_tok, dtype=kind,
                                         stream=torch.cuda.current_stream())
        st["batch"] = binding.CacheBatch(pages, first, lens, n_tokens=n_tok, max_new=max(new), max_len=max(length))
        pool = st["cache"].layer(0)
    else:
        pool = {n: torch.zeros(n_pages, K, page, d, dtype=TYPES[kind], device=DEVICE) for n in ("k", "v")}
        if kind in CODE_MAX:
            pool.update({n: torch.zeros(n_pages, K, page, dtype=torch.float32, device=DEVICE) for n in ("k_scale", "v_scale")})
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
                    codes, scale = _quantise(x, kind)
                    pool[n][lo:hi].view(torch.uint8).copy_(codes.view(torch.uint8))
                    pool[n + "_scale"][lo:hi].copy_(scale)
                else:
                    pool[n][lo:hi].copy_(x)
    st["pool"] = pool
    if case["op"] == "attend":
        st["q"] = torch.randn(n_tok, case["heads"], d, device=DEVICE, generator=g).to(TYPES[case["io"]])
    elif case["op"] == "store":
        # rows of a QKV product: keys and values are slices of wider rows
        qkv = torch.randn(n_tok, (case["heads"] + 2 * K) * d, device=DEVICE, generator=g)
        qkv[:, case["heads"] * d:(case["heads"] + K) * d] *= gain.reshape(-1)
        qkv = qkv.to(TYPES[case["io"]])
        st["k"] = qkv[:, case["heads"] * d:(case["heads"] + K) * d].unflatten(1, (K, d))
        st["v"] = qkv[:, (case["heads"] + K) * d:].unflatten(1, (K, d))
    return st


def _prepare_sample(case, g):
    rows, vocab = case["rows"], case["vocab"]
    rand = lambda: torch.rand(rows, device=DEVICE, generator=g)  # noqa: E731
    st = dict(case=case, logits=case["spread"] * torch.randn(rows, vocab, device=DEVICE, generator=g), uniforms=rand())
    # requests bring their own settings: some use only top-p, some only top-k, some everything, some nothing
    kind = torch.randint(0, 5, (rows,), device=DEVICE, generator=g)
    st["temperature"] = 0.3 + 0.9 * rand()
    st["top_k"] = torch.where((kind == 1) | (kind == 3), torch.randint(1, 101, (rows,), device=DEVICE, generator=g), 0).to(torch.int32)
    st["top_p"] = torch.where((kind == 2) | (kind == 3), 0.3 + 0.69 * rand(), 1.0)
    st["min_p"] = torch.where((kind == 3) | (kind == 4), 0.001 + 0.1 * rand(), 0.0)
    if own:
        from paper_2307_02628_b200 import binding, shapes, synth
        shape = shapes.ModelShape("selection only", 1, 32, 1, 8, vocab, 8, "bf16")
        st["decoder"] = binding.Decoder(shape, synth.make_weights(shape), rows, 4, 4, stream=torch.cuda.current_stream())
    return st


# ---- plain forms -----------------------------------------------------------------------------

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
    x = st["pool"][name][page, :, slot].float()
    return x * st["pool"][name + "_scale"][page, :, slot].unsqueeze(-1) if st["case"]["cache"] in CODE_MAX else x


def _store(st):
    seq, pos = _rows(st)
    page, slot = _slots(st, seq, pos)
    for n in ("k", "v"):
        if st["case"]["cache"] in CODE_MAX:
            codes, scale = _quantise(st[n].float(), st["case"]["cache"])
            st["pool"][n].view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
            st["pool"][n + "_scale"][page, :, slot] = scale
        else:
            st["pool"][n][page, :, slot] = st[n].to(TYPES[st["case"]["cache"]])


def _load(st):
    seq, pos = _rows(st)
    page, slot = _slots(st, seq, pos)
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
    q = torch.zeros(seqs, most, H, d, device=DEVICE)
    q[seq, at] = st["q"].float()
    last = torch.full((seqs, most), -1, device=DEVICE, dtype=torch.long)
    last[seq, at] = pos
    q = q.unflatten(2, (K, H // K)).permute(0, 2, 3, 1, 4).flatten(2, 3)     # [seqs, K, group * most, d]
    k = _values(st, "k", page, slot).transpose(1, 2)                         # [seqs, K, top, d]
    s = (q @ k.transpose(2, 3) * d ** -0.5).unflatten(2, (H // K, most))
    del k
    dead = every > last.unsqueeze(-1)                                        # [seqs, most, top]
    s.masked_fill_(dead[:, None, None], float("-inf"))
    s -= s.amax(-1, keepdim=True)
    s.exp_()
    total = s.sum(-1, keepdim=True)
    o = s.flatten(2, 3) @ _values(st, "v", page, slot).transpose(1, 2)
    o = o.unflatten(2, (H // K, most)) / total
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, at].to(TYPES[case["io"]])


def _sample(st):
    x = st["logits"].double()
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / st["temperature"].double().unsqueeze(1))
    rank = torch.arange(x.shape[1], device=DEVICE)
    top_k = torch.where(st["top_k"] > 0, st["top_k"], x.shape[1]).unsqueeze(1)
    cum = torch.cumsum(w, 1)
    mass = cum.gather(1, (top_k.clamp_max(x.shape[1]) - 1).long())
    before = torch.cat([torch.zeros_like(mass), cum[:, :-1]], 1)
    keep = (rank < top_k) & ((before < st["top_p"].double().unsqueeze(1) * mass) | (st["top_p"].unsqueeze(1) >= 1)) & (w >= st["min_p"].double().unsqueeze(1))
    keep[:, 0] = True
    n = keep.sum(1, keepdim=True)                                           # the three cut the same order, so they leave a prefix
    target = st["uniforms"].double().unsqueeze(1) * cum.gather(1, n - 1)
    j = torch.minimum((cum <= target).sum(1, keepdim=True), n - 1)
    return order.gather(1, j).squeeze(1).to(torch.int32)


def run(st):
    op = st["case"]["op"]
    if not own:
        if op == "store":
            _store(st)
        return _attend(st) if op == "attend" else _sample(st) if op == "sample" else _load(st)
    if op == "sample":
        return st["decoder"].sample(st["logits"], st["uniforms"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
    if op == "attend":
        return st["cache"].attention(0, st["q"], st["batch"])
    if op == "store":
        st["cache"].append(0, st["k"], st["v"], st["batch"])
    k, v = st["cache"].read(0, st["batch"], TYPES[st["case"]["io"]])
    return {"k": k, "v": v}


# ---- the definitions in 64 bits --------------------------------------------------------------

def _round_e4m3(y):
    """To the nearest number with 3 fraction bits, exponents from -6, ties to even, at most 448."""
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "sample":
        return None                                          # a choice, not a computed number
    new, length = _lengths(case)
    K, d, page, kind = case["kv_heads"], case["head_dim"], case["page"], case["cache"]
    out_type = torch.float64
    if case["op"] == "store":
        got = {}
        for n in ("k", "v"):
            x = st[n].double()
            if kind in CODE_MAX:
                scale = (x.abs().amax(-1, keepdim=True) / CODE_MAX[kind]).float().double()      # the cache holds it in 32 bits
                x = (torch.round(x / scale) if kind == "int8" else _round_e4m3(x / scale)) * scale
            else:
                x = x.to(TYPES[kind]).double()
            got[n] = x.to(out_type)
        return got

    def sequence(name, s):
        ids = st["pages"][s, :(length[s] + page - 1) // page].long()
        x = st["pool"][name][ids].double()                    # [pages, K, page, d]
        if kind in CODE_MAX:
            x = x * st["pool"][name + "_scale"][ids].double().unsqueeze(-1)
        return x.transpose(0, 1).reshape(K, -1, d)[:, :length[s]]

    if case["op"] == "load":
        return {n: torch.cat([sequence(n, s).transpose(0, 1) for s in range(len(new))]) for n in ("k", "v")}
    outs = []
    row = 0
    group = case["heads"] // K
    for s, (n, l) in enumerate(zip(new, length)):
        k, v = sequence("k", s), sequence("v", s)
        for lo in range(0, n, 256):
            hi = min(n, lo + 256)
            q = st["q"][row + lo:row + hi].double().reshape(hi - lo, K, group, d)
            p = torch.einsum("nkgd,kjd->kgnj", q, k) / math.sqrt(d)
            hidden = torch.arange(l, device=DEVICE) > torch.arange(l - n + lo, l - n + hi, device=DEVICE).unsqueeze(1)
            p = torch.softmax(p.masked_fill(hidden, float("-inf")), dim=-1)
            outs.append(torch.einsum("kgnj,kjd->nkgd", p, v).reshape(hi - lo, case["heads"], d))
        row += n
    return torch.cat(outs)
