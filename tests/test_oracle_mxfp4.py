"""The 4-bit cache's oracle pinned by arithmetic on the CPU: the levels, the
rounding and the scale rule on values worked out by hand, the places of codes
and scales in a pool block, and the encoder of the input generator (written
apart from it) against it."""

import numpy as np
import pytest

import synth  # noqa: F401
from oracle import attention as oa
from oracle import codecs, kvappend
from synth.attn_inputs import encode_mxfp4, make_batch_from_lengths


def test_levels():
    assert codecs.E2M1_TABLE[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert (codecs.E2M1_TABLE[8:] == -codecs.E2M1_TABLE[:8]).all()


def _row(first, rest=0.0):
    x = np.full(128, rest)
    x[:len(first)] = first
    return x


@pytest.mark.parametrize("a, power", [(1.0, -2), (1.5, -2), (1.7499, -2), (1.75, -1), (1.99, -1), (6.0, 0), (7.0, 1),
                                      (0.0, -125), (2.0 ** -126, -125), (2.0 ** 127 * 1.9, 125)])
def test_scale_of_a_group_follows_its_largest_magnitude(a, power):
    for sign in (1, -1):
        _, byte = codecs.mxfp4_encode(_row([0.0, sign * a]))
        assert byte.tolist() == [power + 127, 2, 2, 2]


def test_codes_round_to_nearest_ties_to_even_and_saturate():
    # the group's scale is 1 (largest magnitude 6.9 < 7)
    x = [6.9, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, -0.0, -0.25, -2.5, -6.5]
    want = [6, 0, 0.5, 1, 0.5, 1, 1.5, 2, 1.5, 2, 3, 4, 3, 4, 6, -0.0, -0.0, -2, -6]
    code, byte = codecs.mxfp4_encode(_row(x))
    assert byte[0] == 127
    got = codecs.E2M1_TABLE[code[:len(x)]]
    assert got.tolist() == want and (np.signbit(got) == np.signbit(want)).all()


def test_groups_are_independent():
    x = np.concatenate([np.full(32, v) for v in (1.0, 100.0, 0.0, -3e-5)])
    code, byte = codecs.mxfp4_encode(x)
    assert len(set(byte.tolist())) == 4
    v = codecs.E2M1_TABLE[code] * np.repeat(2.0 ** (byte.astype(float) - 127), 32)
    assert np.abs(v - x).max() <= 4.0 and np.abs(v[:32] - 1.0).max() == 0.0


def test_places_cover_a_block_once():
    for h_kv in (1, 3):
        for is_v in (False, True):
            codes, scales = set(), set()
            for h in range(h_kv):
                for t in range(16):
                    byte, nib, at = codecs.mxfp4_places(h_kv, h, t, is_v)
                    codes |= set(zip(byte.tolist(), nib.tolist()))
                    scales |= set(at.tolist())
            assert codes == {(b, n) for b in range(h_kv * 1024) for n in (0, 1)}
            assert scales == set(range(h_kv * 1024, h_kv * 1088))


def test_relative_error_of_a_group_is_bounded():
    # a group's largest magnitude is at least 3.5 steps of 2^X and below 7: an element is off by at most half the
    # widest gap, 1 step (between 4 and 6, or from 7 down to 6), so by 1 / 3.5 of the group's largest magnitude
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)) * 5)
    code, byte = codecs.mxfp4_encode(x)
    v = codecs.E2M1_TABLE[code] * np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
    amax = np.abs(x).reshape(500, 4, 32).max(-1)
    assert (np.abs(v - x).reshape(500, 4, 32) <= amax[..., None] / 3.5 + 1e-300).all()


def test_generator_encodes_as_the_oracle_does():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((300, 128)) * np.exp(rng.standard_normal((300, 1)) * 20)).astype(np.float32)
    x[0] = 0.0
    x[1] = -0.0
    x[2, :32] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9] * 4
    x[3] = np.float32(3e38)
    a, b = codecs.mxfp4_encode(x), encode_mxfp4(x)
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()


def test_append_and_pool_filling_agree_and_unused_slots_are_nan():
    """Appending every token of a request writes the pool that the generator
    fills with the same rows, and the attention of an all-equal-keys request is
    the mean of the decoded values."""
    b = make_batch_from_lengths("a", [1, 1], [37, 5], num_q_heads=4, num_kv_heads=2, head_dim=128, q_dtype="bf16",
                                kv_dtype="fp4", out_dtype="bf16", n_pool_blocks=8, seed=3)
    k = oa.materialise_kv(b.k_cache, None, "fp4", b.blocks_of(0), 37)
    v = oa.materialise_kv(b.v_cache, None, "fp4", b.blocks_of(0), 37, is_v=True)
    assert np.isfinite(k).all() and np.isfinite(v).all()
    whole = oa.materialise_kv(b.v_cache, None, "fp4", b.blocks_of(0), 48, is_v=True)
    assert np.isnan(whole[37:]).all()
    # the decoded rows are representable: appending them again changes no value
    from synth.attn_inputs import round_to_bf16_bits
    empty = np.full_like(b.k_cache, 255)
    rows = [round_to_bf16_bits(x.astype(np.float32)) for x in (k, v)]
    k2, v2, _, _ = kvappend.append(empty, empty, None, None, "fp4", rows[0], rows[1], [0, 37], [37], [0, 3], b.blocks_of(0))
    assert (oa.materialise_kv(k2, None, "fp4", b.blocks_of(0), 37) == k).all()
    assert (oa.materialise_kv(v2, None, "fp4", b.blocks_of(0), 37, is_v=True) == v).all()
    out = oa.attend_request(np.zeros((1, 4, 128)), k, v, 4, 2, 1.0)
    assert np.allclose(out[0, 0], v[:, 0].mean(0)) and np.allclose(out[0, 3], v[:, 1].mean(0))
