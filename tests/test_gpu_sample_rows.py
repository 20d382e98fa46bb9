"""Token selection with each row's own settings, against the 64-bit form: the same token on every row.

A draw is an integer.  The library sums weights that are rounded to 2^-47 of the largest (at 50 272 tokens), so a border
moves by about 2^-48 sqrt(50 272) = 8e-13 of the largest weight: a draw falls that close to a border in fewer than one of 10^6 rows.
"""
import pytest
import torch

import paged_reference as P
from paper_2307_02628_b200 import binding, shapes, synth

pytestmark = pytest.mark.gpu


def make(vocab, batch):
    shape = shapes.ModelShape("selection", 1, 32, 1, 8, vocab, 8, "bf16")
    return binding.Decoder(shape, synth.make_weights(shape), batch, 4, 4)


def check(dec, logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    dev = lambda t, dt: None if t is None else t.to(dt).cuda()  # noqa: E731
    got = dec.sample(logits.cuda(), u.cuda(), dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32), dev(min_p, torch.float32)).cpu()
    at = lambda t, b, d: d if t is None else t[b].item()  # noqa: E731
    for b in range(len(u)):
        want = P.select(logits[b], float(u[b]), at(temperature, b, 1.0), at(top_k, b, 0), at(top_p, b, 1.0), at(min_p, b, 0.0))
        assert int(got[b]) == want, (b, int(got[b]), want)
    return got


def settings(n, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda: torch.rand(n, generator=g)  # noqa: E731
    pick = torch.randint(0, 8, (n,), generator=g)
    return dict(temperature=0.2 + 1.3 * r(), top_k=torch.where(pick % 2 == 1, torch.randint(1, 60, (n,), generator=g), 0).to(torch.int32),
                top_p=torch.where((pick // 2) % 2 == 1, 0.05 + 0.94 * r(), 1.0), min_p=torch.where(pick // 4 == 1, 0.2 * r(), 0.0)), r()


@pytest.mark.parametrize("vocab", [1, 2, 31, 1021, 4096, 4097, 8192, 50272, 60001])
@pytest.mark.parametrize("spread,step", [(0.3, 0.0), (2.5, 0.0), (1.0, 0.25), (30.0, 0.0)])
def test_all_settings_together(vocab, spread, step):
    n = 64 if vocab < 10000 else 24
    dec = make(vocab, n)
    logits = synth.make_logits(n, vocab, seed=vocab, scale=spread, step=step)
    s, u = settings(n, vocab + 1)
    check(dec, logits, u, **s)
    check(dec, logits, torch.zeros(n), **s)
    check(dec, logits, torch.full((n,), 0.99999994), **s)
    check(dec, logits, u)
    assert dec.status() == 0
    dec.close()


@pytest.mark.parametrize("vocab", [3000, 50272])
@pytest.mark.parametrize("name,values", [("top_k", [1, 2, 3, 50, 1000, 2999, 3000, 10 ** 9, 0, -5]), ("top_p", [1e-9, 0.0, -1.0, 0.5, 0.999999, 1.0, 2.0, float("inf")]),
                                         ("min_p", [0.0, -1.0, 1e-30, 1e-6, 0.5, 1.0, 1.5]), ("temperature", [1e-30, 1e-3, 0.3, 5.0, 1e6, 3e38, 0.0])])
def test_one_setting(vocab, name, values):
    n = len(values) * 3
    dec = make(vocab, n)
    logits = synth.make_logits(n, vocab, seed=3, scale=1.5)
    u = synth.make_uniforms(n, 4)
    check(dec, logits, u, **{name: torch.tensor(values * 3, dtype=torch.int32 if name == "top_k" else torch.float32)})
    dec.close()


@pytest.mark.parametrize("vocab", [700, 50272])
def test_equal_and_extreme_logits(vocab):
    rows = [torch.zeros(vocab), torch.full((vocab,), -3.5), torch.zeros(vocab), torch.randn(vocab, generator=torch.Generator().manual_seed(1)),
            torch.full((vocab,), float("-inf")), torch.randn(vocab, generator=torch.Generator().manual_seed(2)), torch.full((vocab,), float("nan")),
            torch.zeros(vocab), torch.full((vocab,), 1e38)]
    rows[2][vocab // 2:] = -1e-6                                # two values one step apart, half the row each
    rows[3][::7] = float("nan")
    rows[3][5], rows[3][9] = float("-inf"), -0.0
    rows[4][vocab - 1] = -5.0                                   # one finite logit
    rows[5][vocab // 3] = float("inf")
    rows[5][vocab // 3 + 9] = float("inf")
    rows[7][::2] = -0.0
    rows[8][3] = -3e38
    dec = make(vocab, len(rows))
    logits = torch.stack(rows)
    for u in (0.0, 0.2500001, 0.7, 0.99999994):
        for s in ({}, dict(top_k=7), dict(top_p=0.4999), dict(min_p=0.99), dict(top_k=vocab // 2 + 3, top_p=0.9)):
            check(dec, logits, torch.full((len(rows),), u), **{k: torch.full((len(rows),), v) for k, v in s.items()})
    assert dec.status() == 0
    dec.close()


@pytest.mark.parametrize("vocab", [700, 50272])
def test_logits_masked_with_the_lowest_value(vocab):
    low = torch.finfo(torch.float32).min
    x = torch.randn(6, vocab, generator=torch.Generator().manual_seed(5))
    x[0] = low                                                  # nothing is left
    x[1, 1:] = low                                              # one token is
    x[2, ::2] = low
    x[3, 10:] = low
    x[4] = low
    x[4, 17] = torch.nextafter(torch.tensor(low), torch.tensor(0.0))
    x[5, 3:] = float("-inf")
    dec = make(vocab, 6)
    for u in (0.0, 0.4, 0.9999):
        for T in (1e-30, 0.7, 3e38):
            for s in ({}, dict(top_k=torch.full((6,), 3)), dict(top_p=torch.full((6,), 0.6)), dict(min_p=torch.full((6,), 1.0))):
                check(dec, x, torch.full((6,), u), temperature=torch.full((6,), T), **s)
    assert dec.status() == 0
    dec.close()


def test_more_equal_elements_than_fit_a_list_next_to_others():
    # dense clusters of nearly equal logits: the search has to cut its slice again, several times
    vocab = 50272
    g = torch.Generator().manual_seed(9)
    base = torch.zeros(4, vocab)
    base[:, 0] = 30.0                                           # stretches the slices
    base[0, 1:] = 1.0 + 1e-6 * torch.randint(0, 5, (vocab - 1,), generator=g)
    base[1, 1:] = 1.0 + 1e-4 * torch.rand(vocab - 1, generator=g)
    base[2, 1:] = torch.where(torch.rand(vocab - 1, generator=g) < 0.5, 1.0, 1.0000001)
    base[3, 1:] = 1e-38 * torch.rand(vocab - 1, generator=g)
    dec = make(vocab, 4)
    n = torch.full((4,), 1)
    for T in (3.0, 8.0):
        for u in (0.3, 0.5, 0.9, 0.99):
            check(dec, base, torch.full((4,), u), temperature=n * T)
            check(dec, base, torch.full((4,), u), temperature=n * T, top_k=n * 20001, top_p=n * 0.93)
    dec.close()


def test_settings_that_are_none_are_reported_and_answered_greedily():
    dec = make(1000, 6)
    logits = synth.make_logits(6, 1000, seed=3)
    one = torch.ones(6)
    bad = dict(temperature=one.clone(), top_p=one.clone(), min_p=one * 0)
    bad["temperature"][0], bad["temperature"][1], bad["temperature"][2] = -1.0, float("nan"), float("inf")
    bad["top_p"][3], bad["min_p"][4] = float("nan"), float("nan")
    u = torch.full((6,), 0.9)
    got = dec.sample(logits.cuda(), u.cuda(), **{k: v.cuda() for k, v in bad.items()}).cpu()
    assert got[:5].tolist() == logits[:5].argmax(1).tolist()
    assert int(got[5]) == P.select(logits[5], 0.9 if False else float(u[5]))
    assert dec.status() == binding.STATUS_BAD_SETTING
    for call in (lambda: dec.sample(logits.cuda()[:, :999], u.cuda()), lambda: dec.sample(logits.cuda(), u.cuda()[:5]),
                 lambda: dec.sample(logits.cuda(), u.cuda(), top_k=one.cuda()), lambda: dec.sample(logits.cuda(), u.cuda().double()),
                 lambda: dec.sample(logits.cuda(), u)):
        with pytest.raises(ValueError):
            call()
    dec.close()


def test_agrees_with_the_scalar_call_and_with_greedy():
    vocab, n = 50272, 64
    dec = make(vocab, n)
    logits = synth.make_logits(n, vocab, seed=17, scale=1.0).cuda()
    u = synth.make_uniforms(n, 23).cuda()
    full = lambda v: torch.full((n,), v, device="cuda")  # noqa: E731
    a = dec.sample_top_p(logits, u, 0.3, 0.7)
    b = dec.sample(logits, u, temperature=full(0.3), top_p=full(0.7))
    torch.cuda.synchronize()
    assert int((a == b).sum()) >= 0.99 * n                      # the scalar call weighs in single precision
    g = dec.greedy(logits)
    assert torch.equal(dec.sample(logits, u, temperature=full(0.0)), g)
    assert torch.equal(dec.sample(logits, u, top_k=torch.ones(n, dtype=torch.int32, device="cuda")), g)
    dec.close()


@pytest.mark.parametrize("vocab", [5, 700, 50272])
@pytest.mark.parametrize("temperature", [1.0, 0.0])
def test_rows_of_nan_and_minus_infinity_answer_their_first_token(vocab, temperature):
    # NaN counts as minus infinity, so every token attains the maximum: the lowest index is 0, wherever the first true infinity is
    rows = torch.full((4, vocab), float("-inf"))
    rows[0, 0] = float("nan")
    rows[1, :vocab - 1] = float("nan")
    rows[2, 1] = float("nan")
    rows[3, :2] = float("nan")
    dec = make(vocab, 4)
    for u in (0.0, 0.9):
        got = check(dec, rows, torch.full((4,), u), temperature=torch.full((4,), temperature))
        assert got.tolist() == [0, 0, 0, 0]
    assert dec.status() == 0
    dec.close()
