"""What the planner cuts its row items by: the same beside many tiles with a mask
as without one, and by its prices wherever it prices."""

import os

import numpy as np
import pytest

import paper_2512_04013_amd as aug
from paper_2512_04013_amd.runtime import row_spans

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")

FIELDS = np.dtype([("kvh", "<i2"), ("kind", "i1"), ("stream", "i1"), ("q_row0", "<i4"), ("n_rows", "<i2"), ("stride", "<i2"),
                   ("kb", "<i4"), ("ke", "<i4"), ("pos0", "<i4"), ("bt_off", "<i4"), ("part", "<i4"), ("group", "<i4"),
                   ("notes", "<i4", 3)])


def _plan(shape, q_len, ctx, masked=False):
    q_start = np.concatenate([[0], np.cumsum(q_len)])
    bt = np.concatenate([[0], np.cumsum([-(-c // 16) for c in ctx])])
    first, end = row_spans(q_start, ctx) if masked else (None, None)
    info, plan = aug.aug_attn_plan(shape, q_start, ctx, bt, int(bt[-1]), row_first=first, row_end=end)
    return info, plan[64:64 + 48 * info.num_items].view(FIELDS)


# (query heads, KV heads, head_dim, cache), chunks of rows over earlier tokens, decodes and their median context
BATCHES = [((64, 8, 128, "fp8"), 8, 512, 700, 64, 2000), ((32, 8, 128, "bf16"), 5, 700, 500, 64, 3000),
           ((16, 8, 64, "bf16"), 9, 1000, 300, 48, 4000), ((64, 8, 128, "fp4"), 6, 512, 600, 64, 5000),
           ((32, 8, 128, "fp8"), 12, 400, 600, 200, 1500), ((8, 8, 128, "fp8"), 2, 500, 512, 250, 1000)]


@pytest.mark.parametrize("layer,chunks,rows,prior,decodes,ctx", BATCHES)
def test_causal_spans_cut_the_rows_as_no_spans_do(layer, chunks, rows, prior, decodes, ctx):
    hq, hkv, d, kv = layer
    shape = aug.make_shape(hq, hkv, d, "bf16", kv, "bf16", 0.1)
    rng = np.random.default_rng(decodes)
    q_len = [rows] * chunks + [1] * decodes
    lens = [rows + prior] * chunks + np.clip(rng.lognormal(np.log(ctx), 0.8, decodes), 1, 8 * ctx).astype(int).tolist()
    (info, a), (minfo, b) = _plan(shape, q_len, lens), _plan(shape, q_len, lens, masked=True)
    for f in FIELDS.names[:-1]:
        assert np.array_equal(a[f], b[f]), f
    assert info.num_partials == minfo.num_partials and info.kv_split_tokens == minfo.kv_split_tokens

def test_long_four_bit_contexts_are_cut_by_price_too():
    """Spans over 8192 keys are among the priced ones: 64 contexts of 16384 keys stay
    whole (181 us; two spans of 8192 each: 187), those of 16k to 32k keys go in
    halves (288 and 298 us)."""
    for hq in (8, 32, 64):
        shape = aug.make_shape(hq, 8, 128, "bf16", "fp4", "bf16", 0.1)
        info, items = _plan(shape, [1] * 64, [16384] * 64)
        assert info.num_items == 512 and info.num_partials == 0
        ctx = np.random.default_rng(1).integers(16385, 32769, 64)
        info, items = _plan(shape, [1] * 64, ctx)
        span = items["ke"] - items["kb"]
        assert info.num_items == 1024 and (span > 8192).all() and (span <= 16384).all()
