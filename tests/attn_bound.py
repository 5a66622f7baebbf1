"""Reference rows in float64 and a bound on what the kernels may add to them (no
test functions here).

Where the bound comes from, for one output o = sum p v / sum p of a row:

* a logit's error d: the products' fp32 sum over head_dim is off by at most
  head_dim * 2^-24 * scale * sum |q k| (S below), a few more roundings of the
  logit (times log2 e, minus the maximum, the hardware exp2's last bit) by 32 *
  2^-24 * (1 + |s|), and a tanh cap c, computed from an exp2 and a reciprocal,
  by c * 2^-20. A weight is then off by the factor 1 +- d;
* bf16 and narrower caches: weights are rounded to bf16, 2^-8 of each;
* the fp32 sums over n keys are off by at most n * 2^-24 of their absolute sum;
* numerator and denominator share the weights, so the output moves by at most
  (rel. weight error) * sum p |v - o|, and sum p |v - o| <= sum p |v| + |o|;
* the output's own rounding: 2^-8 |o| (bf16), 2^-24 |o| (fp32).
"""

import numpy as np

from oracle import attention as oa
from oracle.codecs import storage_to_f64
from tests.gpu_util import say


def reference(b, k_cache=None, v_cache=None, k_scale=None, v_scale=None, softcap=0.0, slopes=None, row_first=None,
              row_end=None):
    """(rows [sum_q, H_q, D] float64, elementwise error bound) of a batch."""
    k_cache = b.k_cache if k_cache is None else k_cache
    v_cache = b.v_cache if v_cache is None else v_cache
    k_scale = b.k_scale if k_scale is None else k_scale
    v_scale = b.v_scale if v_scale is None else v_scale
    out = np.zeros((b.total_q, b.num_q_heads, b.head_dim))
    bound = np.zeros_like(out)
    g = b.num_q_heads // b.num_kv_heads
    exact_weights = b.kv_dtype == "f32"
    for r in range(b.num_reqs):
        q0, q1, ctx = int(b.q_start[r]), int(b.q_start[r + 1]), int(b.ctx_len[r])
        k = oa.materialise_kv(k_cache, k_scale, b.kv_dtype, b.blocks_of(r), ctx)
        v = oa.materialise_kv(v_cache, v_scale, b.kv_dtype, b.blocks_of(r), ctx, is_v=True)
        q = storage_to_f64(b.q[q0:q1], b.q_dtype)
        lo = None if row_first is None else row_first[q0:q1]
        hi = None if row_end is None else row_end[q0:q1]
        for h in range(b.num_q_heads):
            p = oa.request_weights(q, k, h, b.num_q_heads, b.num_kv_heads, b.softmax_scale, softcap, slopes, lo, hi)
            vh = v[:, h // g]
            o = p @ vh
            size = (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max(axis=1) * b.softmax_scale     # S
            away = 0.0 if slopes is None else abs(float(slopes[h])) * np.where(p > 1e-12, np.abs(
                ctx - (q1 - q0) + np.arange(q1 - q0)[:, None] - np.arange(ctx)[None, :]), 0).max(axis=1)
            d = 2.0 ** -24 * (b.head_dim * size + 32 * (1 + size + away) + ctx) + softcap * 2.0 ** -20
            rel = d + (0.0 if exact_weights else 2.0 ** -8)
            step = 2.0 ** -24 if exact_weights else 2.0 ** -8
            out[q0:q1, h] = o
            bound[q0:q1, h] = (1.01 * rel)[:, None] * (p @ np.abs(vh) + np.abs(o)) + step * np.abs(o) + 1e-30
    return out, bound


def within(got, want, bound, what=""):
    assert got.shape == want.shape
    assert np.isfinite(got).all(), f"{what}: non-finite outputs"
    worst = float((np.abs(got - want) / bound).max())
    rel = float(np.sqrt(((got - want) ** 2).sum()) / max(np.sqrt((want ** 2).sum()), 1e-30))
    say(f"  {what}: worst error / bound = {worst:.3f}, rel_l2 = {rel:.2e}")
    assert worst <= 1.0, (what, worst)
