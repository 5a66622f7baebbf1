"""Sampling from logits among which signalling NaNs stand, before, beside and behind the largest in
its 16-byte word and in the words that one thread reads: they count as -infinity, as quiet ones do.

Bounds are those of test_gpu_sample.py; tokens and shares are compared with the oracle's row by row."""

import random

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_sample import _check, _run  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BITS = {torch.float32: (torch.int32, (0x7F800001, 0x7FBFFFFF, -0x7FFFFF, 0x7FC00000)),        # the last is a quiet one
        torch.bfloat16: (torch.int16, (0x7F81, 0x7FBF, -0x7F, 0x7FC0))}
SETTINGS = (dict(), dict(temperature=0.0), dict(top_k=1), dict(top_k=2), dict(top_k=40), dict(top_k=1500, top_p=0.9), dict(top_k=3000),
            dict(top_p=0.0), dict(top_p=0.5), dict(top_p=0.95, min_p=0.02), dict(temperature=1e-30), dict(temperature=30.0, top_p=0.7))


def _rows(dtype, vocab, rows, seed):
    """Rows whose largest logit, 9, has a signalling NaN at each place of its word, or in words of the same thread."""
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed)
    word = 4 if dtype == torch.float32 else 8
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2).clamp(max=6).to(dtype)
    integer, kinds = BITS[dtype]
    bits = x.view(integer)
    for r in range(rows):
        at = rng.randrange(vocab)
        x[r, at] = 9.0
        first = at - at % word
        marks = {first + r % word}                                            # in its word
        for turn in range(-4, 5):                                             # 1024 words on: the same thread's next word
            if r % 3 == 1 and turn or r % 3 == 2 and turn == 4 - r % 9:
                marks |= {first + turn * 1024 * word + k for k in (r % word, word - 1)}
        marks |= {rng.randrange(vocab) for _ in range(r % 5)}
        for i in marks - {at}:
            if 0 <= i < vocab:
                bits[r, i] = kinds[rng.randrange(4) if i % 7 == 0 else rng.randrange(3)]
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [2, 4, 8, 13, 300, 2048, 2049, 9000, 40000, 100003])
def test_signalling_nans(dtype, vocab):
    rows, rng = 54, random.Random(vocab)
    say(f"[sample] {vocab} {dtype} with signalling NaNs")
    x = _rows(dtype, vocab, rows, vocab)
    for s in SETTINGS:
        tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
        probs = torch.full((rows,), -7.0, device="cuda")
        got = _check(x, [rng.choice([0.5, rng.random()]) for _ in range(rows)], [s] * rows if s else [{}] * rows, f"{vocab} {s}",
                     tokens=tokens, probs=probs)
        assert all(0 <= t < vocab for t in got)
        chosen = x.float().gather(1, tokens.long()[:, None])
        assert not chosen.isnan().any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_words_of_nans(dtype):
    """The largest alone among signalling NaNs; 1 and 0 among them; and nothing but them."""
    integer, kinds = BITS[dtype]
    for vocab in (4, 8, 5000, 30000):
        x = torch.zeros(3, vocab, device="cuda", dtype=dtype)
        x.view(integer)[:] = kinds[0]
        x[0, vocab - 2] = -4.0
        x[1, 1], x[1, 3] = 1.0, 0.0
        for s, second in ((dict(temperature=0.0), 1), (dict(top_k=2), 1), (dict(top_p=0.9), 1), (dict(top_k=1), 1), (dict(min_p=0.5), 1)):
            tokens, probs = _run(x, [0.5] * 3, [s] * 3)
            assert tokens == [vocab - 2, second, -1] and probs[0] == 1.0 and probs[2] == 0.0, (vocab, s, tokens, probs)
    # of 1 and 0 with weights of 1 and 0.368: the number 0.5 falls into the first, 0.9 into the second
    x = torch.zeros(1, 4, device="cuda", dtype=dtype)
    x.view(integer)[0, 0] = x.view(integer)[0, 2] = kinds[2]
    x[0, 1] = 1.0
    assert [_run(x, [u], [dict(top_k=2)])[0] for u in (0.5, 0.9)] == [[1], [3]]
