"""Modified scores over fp8 blocks whose scales are zero (tokens of zeros) or far
from 1: masked keys stay masked and every score keeps its size. Bounds of
attn_bound.py."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from synth.attn_inputs import make_batch_from_lengths, round_to_bf16_bits  # noqa: E402
from oracle.codecs import bf16_bits_to_f64  # noqa: E402
from tests.attn_bound import reference, within  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

Q, CTX = [1, 40, 1, 129], [300, 90, 64, 400]
SCORES = [dict(softcap=20.0), dict(slopes=True), dict(window=50), dict(softcap=5.0, slopes=True, window=33)]


def _batch(hq, hkv, seed):
    return make_batch_from_lengths("scales", Q, CTX, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, q_dtype="bf16",
                                   kv_dtype="fp8", out_dtype="bf16", n_pool_blocks=sum(-(-c // 16) for c in CTX) + 2, seed=seed,
                                   q_std=2.0)


def _check(b, score, what):
    from paper_2512_04013_amd import runtime as rt
    say(f"[scales] {what} {score}")
    slopes = np.linspace(0.02, 0.3, b.num_q_heads).astype(np.float32) if score.get("slopes") else None
    first, end = rt.row_spans(b.q_start, b.ctx_len, window=score["window"]) if "window" in score else (None, None)
    cap = score.get("softcap", 0.0)
    want, bound = reference(b, softcap=cap, slopes=slopes, row_first=first, row_end=end)
    shape, kv, q, bids = rt.upload_batch(b)
    for split in (0, 64):
        att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=split,
                                row_first=first, row_end=end)
        got = rt.to_host_f64(att.run(q, softcap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda()))
        within(got, want, bound, f"{what} {score} split {split}")


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("score", SCORES, ids=str)
def test_blocks_of_scale_zero(hq, hkv, score):
    b = _batch(hq, hkv, seed=hq)
    rng = np.random.default_rng(1)
    for r in range(b.num_reqs):
        ids = b.blocks_of(r)
        b.k_scale[ids[rng.random(len(ids)) < 0.4]] = 0.0
        b.v_scale[ids[rng.random(len(ids)) < 0.4]] = 0.0
        b.k_scale[ids[-1]] = b.k_scale[ids[0]] = 0.0        # where keys are masked
    _check(b, score, f"zero {hq}/{hkv}")


@pytest.mark.parametrize("hq,hkv", [(2, 2), (16, 2)])
@pytest.mark.parametrize("score", SCORES, ids=str)
def test_large_queries_over_small_scales(hq, hkv, score):
    """Queries 2^100 as large over keys 2^-100 as small have the usual scores."""
    b = _batch(hq, hkv, seed=hq + 1)
    b.q = round_to_bf16_bits((bf16_bits_to_f64(b.q) * 2.0 ** 100).astype(np.float32))
    b.k_scale = (b.k_scale * np.float32(2.0 ** -100)).astype(np.float32)
    _check(b, score, f"small {hq}/{hkv}")
