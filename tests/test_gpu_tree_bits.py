"""Attention of drafts over bf16 caches holds its probabilities to 16 bits: where values of both signs cancel, results
are off by their own rounding and little else.

Bound: that of test_gpu_tree.py with 2^-16 in the place of 2^-8 for a probability (two bf16, each off by half a step,
2^-8, of what it stands for; the row's sum is of the float32 probabilities), and the output's rounding, 2^-8 of it."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402
from oracle import tree as otree  # noqa: E402
from oracle.codecs import storage_to_f64  # noqa: E402
from tests.attn_bound import within  # noqa: E402
from tests.test_gpu_tree import Case  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("layer", [(16, 8, 64, "bf16"), (8, 1, 64, "bf16"), (8, 2, 128, "bf16"), (8, 1, 128, "bf16")])
@pytest.mark.parametrize("rows,ctx", [([5, 1, 64, 17], [40, 900, 130, 17]), ([8, 3], [9000, 2500])])
def test_bits(layer, rows, ctx):
    c = Case(layer, rows, ctx, seed=11)
    got, b = c.run(), c.b
    g = b.num_q_heads // b.num_kv_heads
    masks = [m % (1 << 64) for m in c.t.seen.tolist()]
    small = 0
    for r, (n, length) in enumerate(zip(rows, ctx)):
        q0 = int(b.q_start[r])
        seen = otree.sees(masks[q0:q0 + n], length - n, n)
        k, v = (oa.materialise_kv(x, None, b.kv_dtype, b.blocks_of(r), length, is_v=is_v) for x, is_v in ((b.k_cache, False), (b.v_cache, True)))
        q = storage_to_f64(b.q[q0:q0 + n], b.q_dtype)
        for h in range(b.num_q_heads):
            p = otree.weights(q[:, h], k[:, h // g], seen, b.softmax_scale)
            o, size = p @ v[:, h // g], (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max(1) * b.softmax_scale
            spread = p @ np.abs(v[:, h // g])
            rel = 2.0 ** -24 * (b.head_dim * size + 32 * (1 + size) + length) + 2.0 ** -16
            within(got[q0:q0 + n, h], o, (1.01 * rel)[:, None] * (spread + np.abs(o)) + 2.0 ** -8 * np.abs(o) + 1e-30, f"request {r} head {h}")
            small += int((np.abs(o) < spread / 64).sum())
    assert small > 1000          # results so small beside their terms that an error of 2^-8 in these would show
