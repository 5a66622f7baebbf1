"""The oracle's modified scores, pinned on values worked out by hand."""

import math

import numpy as np

from oracle import attention as oa


def _weights(**kw):
    # three keys, two rows at positions 1 and 2; scores 1, 2, 4 for both rows
    q = np.array([[[1.0, 0.0]], [[1.0, 0.0]]])
    k = np.array([[[1.0, 9.0]], [[2.0, 9.0]], [[4.0, 9.0]]])
    return oa.request_weights(q, k, 0, 1, 1, 1.0, **kw)


def _softmax(*s):
    e = [0.0 if x is None else math.exp(x) for x in s]
    return [x / sum(e) for x in e]


def test_plain_scores_are_the_causal_softmax():
    assert np.allclose(_weights(), [_softmax(1, 2, None), _softmax(1, 2, 4)], rtol=1e-14, atol=0)


def test_cap():
    c = [3 * math.tanh(x / 3) for x in (1, 2, 4)]
    assert np.allclose(_weights(softcap=3.0)[1], _softmax(*c), rtol=1e-14)


def test_bias_by_distance_counts_both_sides():
    w = _weights(slopes=[0.5], end=[3, 3])
    assert np.allclose(w, [_softmax(0.5, 2, 3.5), _softmax(0, 1.5, 4)], rtol=1e-14)


def test_spans_and_rows_without_keys():
    w = _weights(first=[1, 2], end=[3, 2])
    assert np.allclose(w, [_softmax(None, 2, 4), [0, 0, 0]], rtol=1e-14)
    assert not _weights(first=[3, 0], end=[0, 0]).any()


def test_plain_weights_agree_with_the_attention_oracle():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal(s) for s in ((5, 4, 8), (9, 2, 8), (9, 2, 8)))
    want = oa.attend_request(q, k, v, 4, 2, 0.3)
    for h in range(4):
        assert np.allclose(oa.request_weights(q, k, h, 4, 2, 0.3) @ v[:, h // 2], want[:, h], rtol=1e-12)
