"""Scores far beyond the cap, where the tanh is 1 to every bit and only the cap's own
size shows: on the CPU, that the bound used tells a cap that is off by a few per
cent; on the GPU, the kernels against it.

All queries of a KV head point the same way and a key's value is the sign of its
score, so a row's output is (P+ - P-) / (P+ + P-) of the two groups' weights, about
tanh(cap): it moves with the cap and hardly with a single score.

The bound, for o = sum p v / sum p with every weight off by a factor 1 + e: the output
is off by sum p |e| |v - o| / (1 - sum p |e|), plus its own rounding. A raw score x is
off by d = 2^-24 (head_dim * scale * sum |q k| + 32 (1 + |x|)), the capped one by d
times the tanh's largest slope within d of x, at most 2 cap, plus cap * 2^-20 and 32 *
2^-24 * (1 + cap) for its own roundings; e adds 2^-8 for caches whose weights are
rounded to bf16."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402
from oracle.codecs import bf16_bits_to_f64, storage_to_f64  # noqa: E402
from synth.attn_inputs import _write_tokens, make_batch_from_lengths, round_to_bf16_bits  # noqa: E402
from tests.gpu_util import say  # noqa: E402

#          layer, and by how much a cap has to be off to be told (float32 weights and outputs, or bf16 ones)
LAYERS = {"f32-4x4-d64": (4, 4, 64, "f32", 1e-4), "f32-8x2-d128": (8, 2, 128, "f32", 1e-4), "bf16-4x4-d64": (4, 4, 64, "bf16", 0.05),
          "bf16-8x2-d128": (8, 2, 128, "bf16", 0.05), "bf16-8x1-d128": (8, 1, 128, "bf16", 0.05),
          "fp8-8x2-d128": (8, 2, 128, "fp8", 0.05), "fp8-16x2-d128": (16, 2, 128, "fp8", 0.05),
          "fp4-4x4-d128": (4, 4, 128, "fp4", 0.05), "fp4-8x1-d128": (8, 1, 128, "fp4", 0.05)}
Q, CTX = [1, 20, 1, 70], [100, 40, 300, 200]
CAP = 0.5


def _batch(layer, std=3000.0):
    hq, hkv, d, kv, _ = LAYERS[layer]
    io = "f32" if kv == "f32" else "bf16"
    b = make_batch_from_lengths("cap", Q, CTX, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q_dtype=io, kv_dtype=kv,
                                out_dtype=io, n_pool_blocks=sum(-(-c // 16) for c in CTX) + 2, seed=hq + d)
    rng = np.random.default_rng(d)
    g = hq // hkv
    for r in range(b.num_reqs):
        q0, q1, ctx = int(b.q_start[r]), int(b.q_start[r + 1]), int(b.ctx_len[r])
        way = bf16_bits_to_f64(round_to_bf16_bits((rng.standard_normal((hkv, d)) * std).astype(np.float32)))
        size = np.exp2(rng.integers(0, 3, (q1 - q0, hq, 1)))
        q = np.repeat(way, g, axis=0)[None] * size
        b.q[q0:q1] = q if io == "f32" else round_to_bf16_bits(q.astype(np.float32))
        k = oa.materialise_kv(b.k_cache, b.k_scale, kv, b.blocks_of(r), ctx)
        sign = np.sign(np.einsum("thd,hd->th", k, way))
        v = np.repeat(np.where(sign == 0, 1.0, sign)[:, :, None], d, axis=2).astype(np.float32)
        _write_tokens(b.v_cache, b.v_scale, v, b.blocks_of(r), ctx, kv, True)
    return b


def _rows(b, cap):
    """Outputs under `cap` and their bound."""
    out = np.zeros((b.total_q, b.num_q_heads, b.head_dim))
    bound = np.zeros_like(out)
    g = b.num_q_heads // b.num_kv_heads
    fine = b.kv_dtype == "f32"
    for r in range(b.num_reqs):
        q0, q1, ctx = int(b.q_start[r]), int(b.q_start[r + 1]), int(b.ctx_len[r])
        k = oa.materialise_kv(b.k_cache, b.k_scale, b.kv_dtype, b.blocks_of(r), ctx)
        v = oa.materialise_kv(b.v_cache, b.v_scale, b.kv_dtype, b.blocks_of(r), ctx, is_v=True)
        q = storage_to_f64(b.q[q0:q1], b.q_dtype)
        for h in range(b.num_q_heads):
            p = oa.request_weights(q, k, h, b.num_q_heads, b.num_kv_heads, b.softmax_scale, cap)
            x = q[:, h] @ k[:, h // g].T * b.softmax_scale
            d = 2.0 ** -24 * (b.head_dim * b.softmax_scale * (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T) + 32 * (1 + np.abs(x)))
            near = np.maximum(np.abs(x) - d, 0.0)
            e = np.minimum(d / np.cosh(np.minimum(near / cap, 300.0)) ** 2, 2 * cap) + cap * 2.0 ** -20 + 2.0 ** -19 * (1 + cap)
            e = np.expm1(e) + (0.0 if fine else 2.0 ** -8) + ctx * 2.0 ** -24
            vh = v[:, h // g]
            o = p @ vh
            off = np.einsum("jt,jtd->jd", p * e, np.abs(vh[None] - o[:, None])) / (1.0 - (p * e).sum(1, keepdims=True))
            out[q0:q1, h] = o
            bound[q0:q1, h] = off + (2.0 ** -24 if fine else 2.0 ** -8) * (np.abs(o) + off) + 1e-30
    return out, bound


@pytest.mark.parametrize("layer", list(LAYERS))
def test_the_bound_tells_a_wrong_cap(layer):
    b = _batch(layer)
    want, bound = _rows(b, CAP)
    share = LAYERS[layer][4]
    for wrong in (CAP * (1 + share), CAP * (1 - share)):
        got = _rows(b, wrong)[0]
        assert (np.abs(got - want) / bound).max() > 1.2


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("layer", list(LAYERS))
def test_scores_far_beyond_the_cap(layer):
    from paper_2512_04013_amd import runtime as rt
    b = _batch(layer)
    want, bound = _rows(b, CAP)
    shape, kv, q, bids = rt.upload_batch(b)
    for split in (0, 32):
        att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=split)
        got = rt.to_host_f64(att.run(q, softcap=CAP))
        worst = float((np.abs(got - want) / bound).max())
        say(f"[far beyond the cap] {layer} split {split}: worst error / bound {worst:.3f}")
        assert np.isfinite(got).all() and worst <= 1.0
