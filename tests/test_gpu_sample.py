"""Sampling on the GPU against float64 with sums in extended precision, token by token.

Where a row's numbers stay further from every border than what the library may be off,
tokens are equal. Weights are off by a few 2^-52 of each and by half a unit 2^-s each, s >= 42,
so a sum of n of them, at least 1, by less than n * 2^-s; a border by that much on either side,
and the oracle's by 2^-50. MARGIN is that for every row, n being what is not far below the top."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import sampling  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device="cuda")  # noqa: E731
KEYS = ("temperature", "top_k", "top_p", "min_p")


def _run(x, u, settings, **kw):
    from paper_2512_04013_amd import runtime as rt
    args = {k: dev([s[k] for s in settings], torch.int32 if k == "top_k" else torch.float32) for k in KEYS if k in settings[0]}
    tokens, probs = rt.sample(x, dev(u, torch.float32), **args, **kw)
    torch.cuda.synchronize()
    return tokens.tolist(), probs.tolist()


def _check(x, u, settings, what, **kw):
    tokens, probs = _run(x, u, settings, **kw)
    host = x.float().cpu().numpy()
    vocab = x.shape[1]
    margin = vocab * 2.0 ** -min(51, 62 - (vocab - 1).bit_length()) + 2.0 ** -50
    near = 0
    for r, s in enumerate(settings):
        s = {k: float(np.float32(v)) if k != "top_k" else v for k, v in s.items()}
        token, prob, safe = sampling.draw(host[r], float(np.float32(u[r])), **s)
        if safe <= margin:
            # the number 0 lies at a border wherever the first token's share is that small: broad logits
            # of std 6, exp(-22) of the largest and below, have it in a good part of the rows
            near += u[r] != 0.0
            continue
        assert tokens[r] == token, (what, r, s, tokens[r], token, safe)
        # a share: its weight and the sum rounded as above, and once to float32
        assert abs(probs[r] - prob) <= prob * (2.0 ** -24 + margin + 2.0 ** -49), (what, r, probs[r], prob)
    assert near <= max(1, len(settings) // 100), (what, near)      # inputs of the tests stay clear of borders
    return tokens


def _settings(rng, n, vocab, which):
    pick = dict(temperature=lambda: rng.choice([0.0, 0.3, 0.7, 1.0, 1.5, 4.0]),
                top_k=lambda: rng.choice([0, -3, 1, 2, 7, 50, 1000, vocab - 1, vocab, vocab + 5]),
                top_p=lambda: rng.choice([1.0, 0.0, 0.1, 0.5, 0.9, 0.95, 0.999, 2.0]),
                min_p=lambda: rng.choice([0.0, 0.01, 0.05, 0.5, 1.0, 3.0]))
    return [{k: pick[k]() for k in which} for _ in range(n)]


ALL = [(), ("temperature",), ("temperature", "top_k"), ("temperature", "top_p"), ("temperature", "min_p"), ("top_k", "top_p"), KEYS]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows,pad", [(1, 3, 0), (2, 40, 1), (7, 60, 0), (63, 40, 2), (64, 40, 0), (257, 60, 3), (1000, 60, 0), (4099, 40, 5),
                                            (32000, 24, 0), (50257, 16, 47), (131072, 8, 8), (262147, 3, 1), (1 << 20, 2, 0)])
def test_tokens(dtype, vocab, rows, pad):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    rng = random.Random(vocab)
    say(f"[sample] {rows} x {vocab} {dtype}")
    for which in ALL if vocab < 100000 else ALL[-1:]:
        x = torch.randn(rows, vocab + pad, generator=gen, device="cuda") * rng.choice([0.5, 2.0, 6.0])
        x[:, ::97] += torch.rand(rows, len(range(0, vocab + pad, 97)), generator=gen, device="cuda") * 10
        x = x.to(dtype)[:, :vocab]
        u = [rng.choice([0.0, rng.random(), rng.random(), 1 - 2.0 ** -24]) for _ in range(rows)]
        _check(x, u, _settings(rng, rows, vocab, which) if which else [{}] * rows, f"{vocab} {which}")


@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_element(dtype, offset):
    """Rows that begin inside a 16-byte word, with NaN before and behind them."""
    gen = torch.Generator(device="cuda").manual_seed(offset)
    rng = random.Random(offset)
    for vocab in (1, 5, 300, 2049, 5000):
        flat = torch.full((offset + 9 * (vocab + offset),), float("nan"), device="cuda", dtype=dtype)
        x = flat[offset:].view(9, vocab + offset)[:, :vocab]
        x.copy_(torch.randn(9, vocab, generator=gen, device="cuda") * 3)
        _check(x, [rng.random() for _ in range(9)], _settings(rng, 9, vocab, KEYS), f"offset {offset} {vocab}")


def test_borders_by_arithmetic():
    """Equal logits have weights of exactly 1: every border is a whole number."""
    for vocab in (8, 512, 1000, 40000):
        x = torch.full((9, vocab), 3.25, device="cuda")
        u = [0.0, 0.5, 0.25, 1 - 2.0 ** -24, 0.5, 0.5, 0.5, 0.0, 0.75]
        s = [dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) for _ in u]
        s[4]["top_k"], s[5]["top_p"], s[6]["top_p"], s[7]["top_k"] = 4, 0.5, 0.25, 3
        s[8].update(top_k=vocab // 2, top_p=0.5, min_p=1.0)
        tokens, probs = _run(x, u, s)
        want = [0, vocab // 2, vocab // 4, vocab - 1, 2, vocab // 4, vocab // 8, 0, 3 * vocab // 16]
        kept = [vocab] * 4 + [4, vocab // 2, vocab // 4, 3, vocab // 4]
        assert tokens == want, (vocab, tokens, want)
        assert probs == [float(np.float32(1 / n)) for n in kept]


def test_ties_go_to_the_lowest_index():
    """Many equal logits at the cut, in the lowest bits of the key too."""
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((6, 3001), -1.5, device="cuda", dtype=dtype)
        x[:, 7::10] = 2.0
        x[:, 1003] = 2.5
        x[3:, 2999] = -0.0
        x[3:, 5] = 0.0
        hot = [1003] + [i for i in range(7, 3001, 10)]
        u = [0.999999, 0.999999, 0.5, 0.0, 0.99999, 0.3]
        s = [dict(temperature=1.0, top_k=k, top_p=p, min_p=0.0) for k, p in ((20, 1.0), (1, 1.0), (0, 0.3), (302, 1.0), (303, 1.0), (304, 0.99))]
        tokens = _check(x, u, s, f"ties {dtype}")
        # the order begins with 1003 and goes on 7, 17 ...: the last of the 20 by index is 1003
        assert tokens[0] == 1003 and tokens[1] == 1003
        # 301 lie above zero, and zero and minus zero are equal: 302 of the order end with index 5, 303 with 2999,
        # whose share, exp(-2.5) / (1 + 300 exp(-0.5) + 2 exp(-2.5)) = 4.5e-4, the number 0.99999 falls into
        assert len(hot) == 301 and tokens[3] == 5 and tokens[4] == 2999


def test_infinite_and_missing_logits():
    inf, nan = float("inf"), float("nan")
    rows = [[-inf] * 6, [nan] * 6, [-inf, nan, 1.0, -inf, nan, -inf], [inf, 0.0, inf, 5.0, -inf, nan], [0.0, inf, 0.0, 0.0, 0.0, 0.0],
            [nan, 2.0, 2.0, -inf, 2.0, nan], [-3e38, 3e38, -inf, 3e38, 0.0, nan], [1e-45, 0.0, -0.0, -1e-45, -inf, nan]]
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.tensor(rows, device="cuda").to(dtype)
        for s in (dict(), dict(top_k=2), dict(top_p=0.6), dict(min_p=0.9), dict(temperature=0.0), dict(top_k=5, top_p=0.9, min_p=0.2),
                  dict(temperature=1e-30), dict(temperature=1e30)):
            for u in (0.1, 0.7):
                tokens = _check(x, [u] * len(rows), [s] * len(rows) if s else [{}] * len(rows), f"infinite {s}")
                assert tokens[0] == tokens[1] == -1 and tokens[2] == 2 and tokens[4] == 1
    # a signalling NaN
    bits = torch.tensor([[0x7F800001, 0x3F800000, -0x7FFFFF, 0]], dtype=torch.int64).to(torch.int32).cuda()
    assert _run(bits.view(torch.float32), [0.9], [dict(top_k=2)])[0] == [3]


def test_odd_settings():
    """What is not a number, or out of range, means what the definition says."""
    nan = float("nan")
    x = torch.arange(50, 0, -1, device="cuda").float().repeat(9, 1) * 0.01
    s = [dict(temperature=t, top_k=0, top_p=p, min_p=m) for t, p, m in
         ((nan, 1.0, 0.0), (-1.0, 1.0, 0.0), (1.0, nan, nan), (1.0, -2.0, 0.0), (1.0, 7.0, -3.0), (float("inf"), 1.0, 0.0), (1.0, 1.0, 9.0),
          (1.0, 1.0, 0.0), (1.0, 1.0, 0.0))]
    tokens, probs = _run(x, [0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, nan, 2.0], s)
    plain = _run(x[:1], [0.5], [dict(temperature=1.0)])[0][0]
    assert tokens == [0, 0, plain, 0, plain, 25, 0, 0, 49] and probs[0] == probs[6] == 1.0


def test_probabilities_come_out():
    """Frequencies over evenly spread numbers are the shares: each token's count is off by at most one a side."""
    n = 4096
    logits = torch.tensor([0.0, 1.0, 2.0, -1.0, 0.5, -8.0], device="cuda")
    tokens, _ = _run(logits.repeat(n, 1), [(i + 0.5) / n for i in range(n)], [dict(temperature=0.7)] * n)
    share = torch.softmax(logits.double() / float(np.float32(0.7)), 0).cpu().numpy()
    count = np.bincount(tokens, minlength=6)
    assert (np.abs(count - n * share) <= 1.0 + 1e-6).all() and tokens == sorted(tokens)


def test_replays_streams_and_equal_bits():
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows, vocab = 12, 20011
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * 3
    u = torch.rand(rows, generator=gen, device="cuda")
    args = dict(temperature=torch.full((rows,), 0.8, device="cuda"), top_k=torch.full((rows,), 500, dtype=torch.int32, device="cuda"),
                top_p=torch.full((rows,), 0.9, device="cuda"), min_p=torch.full((rows,), 0.001, device="cuda"))
    out = [torch.empty(rows, dtype=t, device="cuda") for t in (torch.int32, torch.float32)]
    rt.sample(x, u, **args, tokens=out[0], probs=out[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rt.sample(x, u, **args, tokens=out[0], probs=out[1])
    side = torch.cuda.Stream()
    for _ in range(4):
        x.normal_(0, 3, generator=gen)
        u.uniform_(0, 1, generator=gen)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = rt.sample(x, u, **args)
        raw = rt.sample(x, u, **args, stream=side.cuda_stream)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(raw[0], want[0])


def test_refusals_and_nothing():
    from paper_2512_04013_amd import runtime as rt
    x, u = torch.zeros(3, 8, device="cuda"), torch.zeros(3, device="cuda")
    for bad in (dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.t()), dict(logits=x.cpu()), dict(uniform=u[:2]), dict(uniform=u.double()),
                dict(temperature=u[:1]), dict(top_k=u), dict(top_p=u.int()), dict(min_p=u.cpu()), dict(tokens=u), dict(probs=u.int())):
        with pytest.raises(ValueError):
            rt.sample(**{"logits": x, "uniform": u, **bad})
    tokens, probs = rt.sample(x[:0], u[:0])
    assert tokens.shape == probs.shape == (0,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("spread", [0.0, 0.03, 3.0])
def test_lists_of_every_size(dtype, spread):
    """Few elements far above the rest, as many as one wave sorts, one more, ..., more than any list holds; equal ones, ones
    within a bin or two, and spread out; cut by number, by weight and by both."""
    rng = random.Random(1)
    gen = torch.Generator(device="cuda").manual_seed(6)
    vocab, sizes = 40000, [1, 2, 63, 64, 65, 100, 127, 128, 129, 255, 257, 300, 1000, 2047, 2048, 2049, 5000]
    x = torch.randn(len(sizes), vocab, generator=gen, device="cuda") - 30
    for r, n in enumerate(sizes):
        at = torch.randperm(vocab, generator=gen, device="cuda")[:n]
        x[r, at] = 5 + spread * torch.rand(n, generator=gen, device="cuda")
    x = x.to(dtype)
    ks = [dict(top_k=n) for n in sizes] + [dict(top_k=n, top_p=0.8) for n in sizes] + [dict(top_k=2 * n, top_p=0.8, min_p=0.3) for n in sizes]
    ps = [dict(top_k=0, top_p=p) for p in (0.05, 0.5, 0.93, 0.999999) for _ in sizes] + [dict(top_k=0, top_p=0.9, min_p=0.6) for _ in sizes]
    settings = [{"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, **s} for s in ks + ps]
    rows = x.repeat(len(settings) // len(sizes), 1)
    u = [rng.random() for _ in settings]
    host, near = rows.float().cpu().numpy(), 0
    tokens, probs = _run(rows, u, settings)
    margin = vocab * 2.0 ** -46 + 2.0 ** -50
    for r, s in enumerate(settings):
        s = {k: float(np.float32(v)) if k != "top_k" else v for k, v in s.items()}
        token, prob, safe = sampling.draw(host[r], float(np.float32(u[r])), **s)
        if safe <= margin:
            near += 1           # equal weights: top_p of n of them may lie at a border, as 0.5 of 64 does
            continue
        assert tokens[r] == token, (r, s, tokens[r], token, safe)
        assert abs(probs[r] - prob) <= prob * (2.0 ** -24 + margin + 2.0 ** -49), (r, s, probs[r], prob)
    say(f"  {near} of {len(settings)} at a border")
    assert near <= len(settings) // (4 if spread == 0.0 else 50)
