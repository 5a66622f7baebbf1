"""Sampling's outputs over what it reads: refused before anything is launched. The addresses are
never used, since every call is refused."""

import ctypes as C

import pytest

import paper_2512_04013_amd as aug

# bytes of 3 rows of 100 float32 logits, 104 apart
READ = dict(logits=(2 * 104 + 100) * 4, uniform=12, temperature=12, top_k=12, top_p=12, min_p=12)


def _call(**kw):
    f = dict(rows=3, vocab=100, dtype=aug.AUG_F32, reserved=0, stride=104)
    f.update({name: (i + 1) << 20 for i, name in enumerate([*READ, "tokens", "probs"])})
    f.update(kw)
    return aug.lib().aug_sample(C.byref(aug.aug_sample_args(**f)), None)


@pytest.mark.parametrize("out", ["tokens", "probs"])
@pytest.mark.parametrize("read", READ)
def test_outputs_over_inputs(out, read):
    at = (list(READ).index(read) + 1) << 20
    for offset in (0, 4, READ[read] - 4, -8):
        assert _call(**{out: at + offset}) == aug.AUG_ERR_INVALID, offset
        assert "overlap" in aug.aug_last_error() and read in aug.aug_last_error()


def test_tokens_over_probs():
    assert _call(tokens=1 << 30, probs=(1 << 30) + 8) == aug.AUG_ERR_INVALID and "overlap" in aug.aug_last_error()
