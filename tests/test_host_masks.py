"""CPU tests of plans with a span of keys for every row, of the score options'
refusals and of the helper that makes spans."""

import os

import numpy as np
import pytest

import paper_2512_04013_amd as aug
from paper_2512_04013_amd import AugError
from tests.test_host_abi import _decode_plan  # noqa: F401  (the image's layout)

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")

SHAPES = {"f32": (4, 4, 64), "bf16": (32, 8, 128), "fp8": (64, 8, 128), "fp4": (16, 8, 128)}


def _shape(kv="bf16"):
    hq, hkv, d = SHAPES[kv]
    io = "f32" if kv == "f32" else "bf16"
    return aug.make_shape(hq, hkv, d, io, kv, io, 0.1)


def _items(plan, info):
    """Items and merge groups of an image that may end with row spans."""
    base = plan[:len(plan) - (-(-info.total_rows * 8 // 16) * 16)]
    hdr, items, groups = _decode_plan(base)
    spans = plan[len(base):].view(np.int32)[:2 * info.total_rows].reshape(-1, 2)
    return items, groups, spans


def _random_spans(rng, q_len, ctx):
    first, end = [], []
    for q, c in zip(q_len, ctx):
        pos = np.arange(c - q, c)
        kind = rng.integers(0, 5)
        lo, hi = np.zeros(q, int), pos + 1
        if kind == 1:
            lo = np.maximum(0, pos - int(rng.integers(0, 100)))
        elif kind == 2:
            hi = np.maximum(hi, int(rng.integers(0, c + 1)))
        elif kind == 3:
            lo, hi = np.sort(rng.integers(0, c + 1, (2, q)), axis=0)
        elif kind == 4:
            lo, hi = hi, lo
        first.append(lo)
        end.append(hi)
    return np.concatenate(first), np.concatenate(end)


@pytest.mark.parametrize("kv", list(SHAPES))
@pytest.mark.parametrize("split", [0, 32, 256])
def test_masked_plans_cover_every_seen_key_once(kv, split):
    rng = np.random.default_rng(split + len(kv))
    s = _shape(kv)
    for trial in range(12):
        n = int(rng.integers(1, 12))
        q_len = np.where(rng.random(n) < 0.5, rng.integers(2, 200, n), 1)
        ctx = q_len + rng.integers(0, int(rng.choice([20, 3000])), n)
        q_start = np.concatenate([[0], np.cumsum(q_len)])
        bt = np.concatenate([[0], np.cumsum(-(-ctx // 16))])
        first, end = _random_spans(rng, q_len, ctx)
        info, plan = aug.aug_attn_plan(s, q_start, ctx, bt, int(bt[-1]), np.arange(bt[-1]), kv_split_tokens=split,
                                       row_first=first, row_end=end)
        items, groups, spans = _items(plan, info)
        assert (spans[:, 0] == first).all() and (spans[:, 1] == end).all()
        cover, slots = {}, {}
        for it in items:
            kb, ke, pos0 = int(it["kb"]), int(it["ke"]), int(it["pos0"])
            r = int(np.searchsorted(q_start, it["q_row0"], side="right") - 1)
            assert it["bt_off"] == bt[r] and 0 <= kb and ke <= ctx[r] and kb % (64 if it["kind"] else 16) == 0
            for j in range(int(it["n_rows"])):
                row = int(it["q_row0"]) + j
                assert pos0 + j == ctx[r] - q_len[r] + row - q_start[r]
                cover.setdefault((row, int(it["kvh"])), []).append((kb, ke))
                if it["part"] >= 0:
                    slot = int(it["part"]) + j * int(it["stride"])
                    assert slot not in slots
                    slots[slot] = (row, int(it["kvh"]))
                    q_row, g_kvh, part0, parts = groups[int(it["group"]) + j]
                    assert (q_row, g_kvh) == (row, it["kvh"]) and part0 <= slot < part0 + parts
                if it["kind"]:
                    lo, hi = it["res2"][0], it["res2"][1]
                    assert lo >= hi or (first[row] <= lo and hi <= end[row])
        assert set(slots) == set(range(info.num_partials))
        for row in range(int(q_start[-1])):
            for h in range(s.num_kv_heads):
                spans_ = sorted(cover[(row, h)])
                assert all(a[1] == c[0] for a, c in zip(spans_, spans_[1:]))
                if end[row] > first[row]:
                    assert spans_[0][0] <= first[row] and spans_[-1][1] >= end[row]
        ws = info.num_partials and info.workspace_bytes
        assert (ws > 0) == (info.num_partials > 0)


def test_causal_spans_plan_the_causal_work():
    """Spans that say what the causal mask says give the same items, but for the
    notes of the tiles, and a window takes the work that it leaves."""
    from paper_2512_04013_amd.runtime import row_spans
    s = _shape()
    q_start, ctx, bt = [0, 1, 301, 302], [5000, 700, 40], [0, 313, 357, 360]
    info, plan = aug.aug_attn_plan(s, q_start, ctx, bt, 400)
    first, end = row_spans(q_start, ctx)
    minfo, mplan = aug.aug_attn_plan(s, q_start, ctx, bt, 400, row_first=first, row_end=end)
    _, a, _ = _decode_plan(plan)
    b, _, _ = _items(mplan, minfo)
    for f in ("kvh", "kind", "q_row0", "n_rows", "stride", "kb", "ke", "pos0", "bt_off", "part", "group"):
        assert (a[f] == b[f]).all(), f
    only_end, _ = aug.aug_attn_plan(s, q_start, ctx, bt, 400, row_end=end)
    assert only_end.plan_bytes == minfo.plan_bytes > info.plan_bytes
    first, end = row_spans(q_start, ctx, window=64)
    winfo, wplan = aug.aug_attn_plan(s, q_start, ctx, bt, 400, row_first=first, row_end=end)
    w, _, _ = _items(wplan, winfo)
    decode = w[w["q_row0"] == 0]
    assert (decode["kb"] == 4928).all() and (decode["ke"] == 5000).all() and winfo.num_partials == 0


def test_bad_spans_are_refused():
    s = _shape()
    q_start, ctx, bt = [0, 1, 4], [20, 30], [0, 2, 4]
    ok = np.array([0, 0, 0, 0]), np.array([20, 28, 29, 30])

    def plan(first=ok[0], end=ok[1], **kw):
        return aug.aug_attn_plan(s, q_start, ctx, bt, 4, row_first=first, row_end=end, **kw)

    plan()
    plan(first=np.array([20, 30, 5, 30]), end=np.array([0, 0, 4, 30]))        # rows that see nothing
    for name, row, value in (("first", 0, -1), ("first", 0, 21), ("end", 0, 21), ("end", 3, 31), ("end", 2, -1),
                             ("first", 1, 2 ** 31 - 1), ("end", 1, -2 ** 31)):
        a = ok[name == "end"].copy()
        a[row] = value
        with pytest.raises(AugError) as e:
            plan(**{name: a})
        assert e.value.status == aug.AUG_ERR_INVALID and f"row {row if row == 0 else row - 1} of" in str(e.value)
    for a in (np.zeros(3, int), np.zeros(5, int), np.zeros((4, 1), int)):
        with pytest.raises(ValueError):
            plan(first=a)
    s8 = _shape("fp8")
    for path in (aug.AUG_TILES_FP8_QK, aug.AUG_TILES_FP8):
        with pytest.raises(AugError) as e:
            aug.aug_attn_plan(s8, q_start, ctx, bt, 4, row_first=ok[0], tile_path=path)
        assert e.value.status == aug.AUG_ERR_UNSUPPORTED
    info, _ = aug.aug_attn_plan(s, [0], [], [0], 4, row_first=[], row_end=[])
    assert info.num_items == 0


def test_score_options_are_checked():
    L, s = aug.lib(), _shape()
    info, _ = aug.aug_attn_plan(s, [0, 1, 41], [700, 300], [0, 44, 63], 70)

    def call(score, shape=s, info=info, plan=16, ws=16, ws_bytes=1 << 40):
        return L.aug_attn_mixed_scored(aug.C.byref(shape), aug.C.byref(info), score, plan, 16, 16, 16, 16, 16, 16, 70,
                                       16, ws, ws_bytes, None)

    Opt = aug.aug_score_options
    assert call(None) == aug.AUG_ERR_INVALID
    assert call(aug.C.byref(Opt(0.0, 1, None))) == aug.AUG_ERR_INVALID
    for cap in (-1.0, 0.0009, 4097.0, float("inf"), float("nan")):
        assert call(aug.C.byref(Opt(cap, 0, None))) == aug.AUG_ERR_INVALID and "softcap" in aug.aug_last_error()
    good = aug.C.byref(Opt(50.0, 0, None))
    assert call(good, plan=None) == aug.AUG_ERR_INVALID and "NULL" in aug.aug_last_error()
    split, _ = aug.aug_attn_plan(s, [0, 1], [700], [0, 44], 70, kv_split_tokens=64)
    assert call(good, info=split, ws=None, ws_bytes=0) == aug.AUG_ERR_NO_SPACE
    s8 = _shape("fp8")
    info8, _ = aug.aug_attn_plan(s8, [0, 1, 41], [700, 300], [0, 44, 63], 70, tile_path=aug.AUG_TILES_FP8)
    assert call(good, shape=s8, info=info8) == aug.AUG_ERR_UNSUPPORTED
    # a plan image whose size is neither with nor without spans
    bad = aug.aug_attn_plan_info.from_buffer_copy(info)
    bad.plan_bytes += 16
    assert call(good, info=bad) == aug.AUG_ERR_INVALID and "consistent" in aug.aug_last_error()
    empty, _ = aug.aug_attn_plan(s, [0], [], [0], 70)
    assert call(good, info=empty, plan=None) == aug.AUG_OK


def test_row_spans():
    from paper_2512_04013_amd.runtime import row_spans
    q_start, ctx = [0, 3, 4], [5, 9]
    first, end = row_spans(q_start, ctx)
    assert first.tolist() == [0, 0, 0, 0] and end.tolist() == [3, 4, 5, 9]
    first, end = row_spans(q_start, ctx, window=2)
    assert first.tolist() == [1, 2, 3, 7] and end.tolist() == [3, 4, 5, 9]
    first, end = row_spans(q_start, ctx, prefix_len=[4, 100])
    assert first.tolist() == [0, 0, 0, 0] and end.tolist() == [4, 4, 5, 9]
    first, end = row_spans(q_start, ctx, window=3, doc_start=[2, 2, 4, 0])
    assert first.tolist() == [2, 2, 4, 6] and end.tolist() == [3, 4, 5, 9]


def test_tiles_end_where_no_row_sees_a_key():
    """Rows of two documents with padding between them do not share a tile, and the
    tiles' notes name the first key that a row sees."""
    s = _shape()
    ctx = 400
    pos = np.arange(ctx)
    first, end = np.where(pos < 110, 0, 150), pos + 1
    end[110:150] = 0                                    # padding sees nothing, and nobody sees it
    info, plan = aug.aug_attn_plan(s, [0, ctx], [ctx], [0, 25], 25, row_first=first, row_end=end)
    items, _, _ = _items(plan, info)
    for it in items[items["kvh"] == 0]:
        rows = np.arange(it["q_row0"], it["q_row0"] + it["n_rows"])
        live = rows[end[rows] > first[rows]]
        if len(live):
            assert (live < 110).all() or (live >= 150).all()
            assert it["res2"][2] == first[live].min() and it["kb"] == it["res2"][2] // 64 * 64


def test_malformed_batches_are_refused_before_their_spans_are_read():
    """q_start that does not rise is refused, although spans of its last entry's
    length were given: no span beyond them is looked at."""
    s = _shape()
    spans = np.zeros(5, np.int32)
    for q_start in ([0, 1000000, 5], [0, 5, 5], [0, 7, 5]):
        with pytest.raises(AugError) as e:
            aug.aug_attn_plan(s, q_start, [1000000, 40], [0, 62500, 62503], 62503, row_first=spans, row_end=spans)
        assert e.value.status == aug.AUG_ERR_INVALID and "rows" in str(e.value)
    with pytest.raises(ValueError):
        aug.aug_attn_plan(s, [0, 1], [40], [0, 3], 3, row_first=np.array([2 ** 32 + 1]))
