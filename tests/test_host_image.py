"""The plan image's parts lie where include/aug.h says: header, items, merge groups,
counters, append items, and the spans of a plan with a mask at its end."""

import os

import numpy as np
import pytest

import paper_2512_04013_amd as aug

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
@pytest.mark.parametrize("masked", [False, True])
def test_counters_stand_between_the_groups_and_the_append_items(kv, masked):
    s = aug.make_shape(16, 8, 128, "bf16", kv, "bf16", 0.1)
    q_start, ctx, bt = [0, 1, 41, 42], [700, 300, 90], [0, 44, 63, 69]
    first, end = np.zeros(42, np.int32), np.concatenate([[700], np.arange(261, 301), [90]]).astype(np.int32)
    span = dict(row_first=first, row_end=end) if masked else {}
    info, plan = aug.aug_attn_plan(s, q_start, ctx, bt, 70, kv_split_tokens=64, **span)
    assert info.num_merge_groups > 0
    at = 64 + 48 * info.num_items + 16 * info.num_merge_groups
    behind = at + 4 * info.num_merge_groups
    assert plan[:64].view(np.int32)[10] == at and not plan[at:behind].any()
    groups = plan[at - 16 * info.num_merge_groups:at].view(np.int32).reshape(-1, 4)
    assert groups[:, 3].min() > 1 and groups[:, 3].sum() == info.num_partials
    append = -(-behind // 16) * 16
    items = plan[append:append + 16 * info.num_append_items].view(np.int32).reshape(-1, 4)
    assert items[0].tolist() == [0, 1 + (699 % 16 << 16), 43, 0]
    rest = plan[append + 16 * info.num_append_items:]
    if masked:
        assert np.array_equal(rest.view(np.int32).reshape(-1, 2)[:42], np.stack([first, end], 1))
    else:
        assert rest.size == 0
