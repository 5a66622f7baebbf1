"""Modified scores on the GPU, through the C ABI, over every cache format:
capped scores, bias by distance, a span of keys for every row, all together, for
decode rows, prefill rows and tiles, whole and split, against float64 within an
elementwise bound."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import synth  # noqa: E402
from oracle import kvappend  # noqa: E402
from synth.attn_inputs import make_batch_from_lengths  # noqa: E402
from tests.attn_bound import reference, within  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

LAYERS = {"f32-4x4-d64": (4, 4, 64, "f32"), "f32-8x2-d128": (8, 2, 128, "f32"), "f32-8x1-d128": (8, 1, 128, "f32"),
          "bf16-16x8-d64": (16, 8, 64, "bf16"), "bf16-8x1-d64": (8, 1, 64, "bf16"), "bf16-4x4-d128": (4, 4, 128, "bf16"),
          "bf16-32x8-d128": (32, 8, 128, "bf16"), "bf16-16x2-d128": (16, 2, 128, "bf16"),
          "fp8-16x8-d128": (16, 8, 128, "fp8"), "fp8-8x2-d128": (8, 2, 128, "fp8"), "fp8-16x2-d128": (16, 2, 128, "fp8"),
          "fp4-4x4-d128": (4, 4, 128, "fp4"), "fp4-8x2-d128": (8, 2, 128, "fp4"), "fp4-16x2-d128": (16, 2, 128, "fp4")}
SCORES = [dict(softcap=30.0), dict(slopes=True), dict(mask="window"), dict(mask="documents"), dict(mask="prefix"),
          dict(mask="random"), dict(softcap=5.0, slopes=True, mask="window")]


def _batch(layer, q_lens, ctx_lens, seed=0, **kw):
    hq, hkv, d, kv = LAYERS[layer]
    io = "f32" if kv == "f32" else "bf16"
    return make_batch_from_lengths("s", q_lens, ctx_lens, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q_dtype=io,
                                   kv_dtype=kv, out_dtype=io, n_pool_blocks=sum(-(-c // 16) for c in ctx_lens) + 4,
                                   seed=seed, **kw)


def _spans(b, mask, seed=0):
    rng = np.random.default_rng(seed)
    first, end = [], []
    for r in range(b.num_reqs):
        q, ctx = int(b.q_len[r]), int(b.ctx_len[r])
        pos = np.arange(ctx - q, ctx)
        lo, hi = np.zeros(q, int), pos + 1
        if mask == "window":
            lo = np.maximum(0, pos - [0, 1, 16, 40, 100][r % 5] + 1)      # a window of 0 keys sees none
            hi = np.where(lo > pos, lo, hi)
        elif mask == "prefix":
            hi = np.maximum(hi, min(ctx, [0, 5, 64, 1000][r % 4]))
        elif mask == "documents":
            starts = np.unique(np.concatenate([[0], rng.integers(0, ctx, max(1, ctx // 30))]))
            doc = np.searchsorted(starts, pos, side="right") - 1
            lo = starts[doc]
            hi = np.where(doc % 4 == 3, 0, hi)                            # padding sees nothing
        elif mask == "random":
            lo, hi = np.sort(rng.integers(0, ctx + 1, (2, q)), axis=0)
        first.append(lo)
        end.append(hi)
    return np.concatenate(first).astype(np.int32), np.concatenate(end).astype(np.int32)


def _slopes(b):
    return np.array([2.0 ** (-4.0 * (h + 1) / b.num_q_heads) for h in range(b.num_q_heads)], np.float32)


def _check(b, score, splits=(0,), what="", spans=None, seed=0):
    from paper_2512_04013_amd import runtime as rt
    first, end = spans or (_spans(b, score["mask"], seed) if "mask" in score else (None, None))
    slopes = _slopes(b) if score.get("slopes") else None
    cap = score.get("softcap", 0.0)
    want, bound = reference(b, softcap=cap, slopes=slopes, row_first=first, row_end=end)
    shape, kv, q, bids = rt.upload_batch(b)
    dev = None if slopes is None else torch.from_numpy(slopes).cuda()
    for split in splits:
        att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=split,
                                row_first=first, row_end=end)
        att.out.fill_(float("nan"))
        got = rt.to_host_f64(att.run(q, softcap=cap, slopes=dev))
        torch.cuda.synchronize()
        within(got, want, bound, f"{what} {score} split {split}")
        if first is not None:
            assert not got[np.asarray(first) >= np.asarray(end)].any(), "rows that see no key are zero"
    return att


@pytest.mark.parametrize("layer", list(LAYERS))
@pytest.mark.parametrize("score", SCORES, ids=lambda s: "-".join(f"{k}={v}" for k, v in s.items()))
def test_rows_and_tiles(layer, score):
    say(f"[scored] {layer} {score}")
    std = 6.0 if "softcap" in score else 1.0
    b = _batch(layer, [1, 1, 40, 1, 1, 129, 1, 2], [1, 700, 90, 64, 17, 300, 2100, 2], seed=len(layer), q_std=std)
    _check(b, score, (0, 32), layer)


@pytest.mark.parametrize("layer", ["bf16-32x8-d128", "fp8-16x2-d128", "fp4-8x2-d128", "f32-8x2-d128"])
@pytest.mark.parametrize("score", SCORES, ids=lambda s: "-".join(f"{k}={v}" for k, v in s.items()))
def test_decodes_alone(layer, score):
    say(f"[scored decodes] {layer} {score}")
    ctx = [1, 2, 15, 16, 17, 33, 100, 257, 1111, 2500]
    b = _batch(layer, [1] * len(ctx), ctx, seed=3, q_std=4.0 if "softcap" in score else 1.0)
    _check(b, score, (0, 16, 64), layer)


@pytest.mark.parametrize("layer", ["bf16-8x1-d64", "f32-8x1-d128", "fp4-16x2-d128", "fp8-16x2-d128", "bf16-16x2-d128"])
def test_long_split_tiles_and_rows(layer):
    say(f"[scored long] {layer}")
    for score in (dict(softcap=20.0, slopes=True), dict(mask="random"), dict(slopes=True, mask="documents")):
        b = _batch(layer, [33, 1], [9000, 9001], seed=8, q_std=3.0)
        _check(b, score, (0,), layer)


def test_no_row_sees_a_key():
    for layer in ("bf16-32x8-d128", "fp4-8x2-d128", "f32-4x4-d64", "fp8-8x2-d128"):
        b = _batch(layer, [40, 1, 3], [50, 17, 3])
        none = np.full(b.total_q, 3, np.int32)
        att = _check(b, dict(mask="none"), what=layer, spans=(none, none))
        assert not att.out.any()


@pytest.mark.parametrize("layer", ["bf16-32x8-d128", "fp8-16x2-d128", "fp4-16x2-d128", "f32-8x2-d128"])
def test_without_modifiers_the_plain_results(layer):
    """Causal spans and no cap and no bias give what the plain launch gives, up to
    the last rounding; the noalloc entry takes a masked plan too."""
    from paper_2512_04013_amd import AUG_OK, aug_attn_mixed_noalloc, lib, aug_score_options, C
    from paper_2512_04013_amd import runtime as rt
    b = _batch(layer, [1, 33, 1], [500, 60, 40], seed=5)
    want, bound = reference(b)
    shape, kv, q, bids = rt.upload_batch(b)
    first, end = rt.row_spans(b.q_start, b.ctx_len)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=64,
                            row_first=first, row_end=end)
    a = att.run(q).clone()
    within(rt.to_host_f64(a), want, bound, layer)
    att.out.zero_()
    aug_attn_mixed_noalloc(shape, att.info, att.plan_dev, q, kv.k_cache, kv.v_cache, kv.k_scale, kv.v_scale, bids,
                           kv.num_pool_blocks, att.out)
    assert torch.equal(att.out, a)
    plain = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=64)
    p = lambda t: None if t is None else t.data_ptr()
    score = aug_score_options(0.0, 0, None)
    st = lib().aug_attn_mixed_scored(C.byref(shape), C.byref(plain.info), C.byref(score), p(plain.plan_dev), p(q),
                                     p(kv.k_cache), p(kv.v_cache), p(kv.k_scale), p(kv.v_scale), p(bids),
                                     kv.num_pool_blocks, p(plain.out), p(plain.workspace), plain.workspace.numel(),
                                     torch.cuda.current_stream().cuda_stream)
    assert st == AUG_OK
    within(rt.to_host_f64(plain.out), want, bound, layer + " unmasked")


@pytest.mark.parametrize("cap", [0.0009765625, 0.5, 4096.0])
@pytest.mark.parametrize("layer", ["bf16-32x8-d128", "f32-8x2-d128", "fp4-8x2-d128"])
def test_caps_at_the_ends_of_their_range(layer, cap):
    b = _batch(layer, [1, 40], [300, 90], seed=6, q_std=8.0)
    _check(b, dict(softcap=cap), what=layer)


def test_scores_far_beyond_the_cap():
    # logits of thousands: tanh is 1 to every bit, all keys with a positive score weigh the same
    for layer in ("bf16-32x8-d128", "f32-4x4-d64", "fp8-8x2-d128"):
        b = _batch(layer, [1, 20], [100, 40], seed=7, q_std=3000.0)
        _check(b, dict(softcap=2.0), what=layer)


def test_negative_slopes_and_unaligned_slopes():
    """Slopes may favour far keys, and need no alignment but a float's."""
    from paper_2512_04013_amd import runtime as rt
    b = _batch("bf16-32x8-d128", [1, 33], [120, 60], seed=10)
    slopes = np.linspace(-0.2, 0.3, 32).astype(np.float32)
    want, bound = reference(b, slopes=slopes)
    shape, kv, q, bids = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids)
    room = torch.zeros(35, device="cuda")
    room[3:] = torch.from_numpy(slopes).cuda()
    within(rt.to_host_f64(att.run(q, slopes=room[3:])), want, bound, "slopes")
    for bad in (room[:32].double(), room[:31], room[3:].cpu(), room.repeat(2)[::2][:32]):
        with pytest.raises(ValueError):
            att.run(q, slopes=bad)


def test_distances_from_far_positions_keep_their_precision():
    """A row whose keys all lie far behind its position: the bias there is in the
    thousands, its differences between keys are what counts."""
    b = _batch("f32-8x2-d128", [1, 3], [9000, 9000], seed=12)
    first = np.array([10, 100, 0, 4000], np.int32)
    end = np.array([60, 164, 5, 4100], np.int32)
    from paper_2512_04013_amd import runtime as rt
    slopes = np.linspace(0.1, 0.9, 8).astype(np.float32)
    want, bound = reference(b, slopes=slopes * 1.0, row_first=first, row_end=end)
    near = reference(b, slopes=None, row_first=first, row_end=end)[1]
    shape, kv, q, bids = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, row_first=first, row_end=end)
    got = rt.to_host_f64(att.run(q, slopes=torch.from_numpy(slopes).cuda()))
    within(got, want, np.minimum(bound, 4 * near), "far rows")


@pytest.mark.parametrize("layer", ["bf16-32x8-d128", "fp4-16x2-d128"])
def test_a_step_with_modified_scores_in_a_graph(layer):
    """Append and masked, capped, biased attention of two layers that share a plan,
    eager and captured: every replay equals the eager result and float64; new
    slopes are read by the next replay."""
    from paper_2512_04013_amd import runtime as rt
    say(f"[scored step] {layer}")
    b = synth.poison_new_slots(_batch(layer, [1, 40, 1, 1], [700, 90, 33, 1], seed=14, q_std=4.0))
    k_new, v_new = synth.make_new_kv(b, seed=15)
    first, end = _spans(b, "window")
    slopes = _slopes(b)
    shape, kv, q, bids = rt.upload_batch(b)
    _, kv2, _, _ = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=64,
                            row_first=first, row_end=end)
    kd, vd = rt.to_device_array(k_new, "bf16", "cuda"), rt.to_device_array(v_new, "bf16", "cuda")
    sl = torch.from_numpy(slopes).cuda()
    out2 = torch.empty_like(att.out)

    def step():
        for pool, out in ((kv, att.out), (kv2, out2)):
            att.append(kd, vd, kv=pool)
            att.run(q, kv=pool, out=out, softcap=30.0, slopes=sl)

    step()
    torch.cuda.synchronize()
    eager = att.out.clone()
    k, v, ks, vs = kvappend.append(b.k_cache, b.v_cache, b.k_scale, b.v_scale, b.kv_dtype, k_new, v_new, b.q_start,
                                   b.ctx_len, b.bt_start, b.block_ids)
    want, bound = reference(b, k, v, ks, vs, softcap=30.0, slopes=slopes, row_first=first, row_end=end)
    within(rt.to_host_f64(eager), want, bound, "eager")
    assert torch.equal(out2, eager)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    for i in range(3):
        att.out.zero_()
        out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(att.out, eager) and torch.equal(out2, eager)
        step()
        torch.cuda.synchronize()
    sl.zero_()
    graph.replay()
    torch.cuda.synchronize()
    want, bound = reference(b, k, v, ks, vs, softcap=30.0, row_first=first, row_end=end)
    within(rt.to_host_f64(att.out), want, bound, "new slopes")


@pytest.mark.parametrize("layer", ["f32-4x4-d64", "bf16-16x8-d64", "bf16-32x8-d128", "fp8-16x2-d128", "fp4-8x2-d128"])
@pytest.mark.parametrize("mask", ["window", "padding", "far"])
def test_keys_that_no_row_sees_may_hold_anything(layer, mask):
    """NaN keys, values and scales wherever no row of the request looks: before a
    window, between documents, behind a prefix. The results are those without."""
    from paper_2512_04013_amd import runtime as rt
    say(f"[scored NaN] {layer} {mask}")
    b = _batch(layer, [1, 1, 140, 60, 2], [300, 77, 500, 333, 100], seed=16)
    first, end = [], []
    for r in range(b.num_reqs):
        q, ctx = int(b.q_len[r]), int(b.ctx_len[r])
        pos = np.arange(ctx - q, ctx)
        lo, hi = np.zeros(q, int), pos + 1
        if mask == "window":
            lo = np.maximum(0, pos - 37)
        elif mask == "padding":
            lo = np.where(pos % 70 < 50, pos // 70 * 70, ctx)             # documents of 50 rows, 20 of padding
            hi = np.where(pos % 70 < 50, pos + 1, 0)
        else:
            lo, hi = np.full(q, ctx // 3), np.full(q, ctx // 2)
        first.append(lo)
        end.append(hi)
    first, end = np.concatenate(first).astype(np.int32), np.concatenate(end).astype(np.int32)
    slopes = _slopes(b)
    want, bound = reference(b, softcap=20.0, slopes=slopes, row_first=first, row_end=end)
    h = b.num_kv_heads
    for r in range(b.num_reqs):
        seen = np.zeros(int(b.ctx_len[r]), bool)
        for row in range(int(b.q_start[r]), int(b.q_start[r + 1])):
            seen[first[row]:end[row]] = True
        for t in np.nonzero(~seen)[0]:
            blk, slot = b.blocks_of(r)[t // 16], t % 16
            if b.kv_dtype == "fp4":
                b.k_cache[blk, h * 1024:].reshape(h, 16, 4)[:, slot] = 255
                b.v_cache[blk, h * 1024:].reshape(h, 4, 16)[:, :, slot] = 255
            else:
                nan = {"f32": np.float32(np.nan), "bf16": np.uint16(0x7FC0), "fp8": np.uint8(0x7F)}[b.kv_dtype]
                b.k_cache[blk, :, slot] = nan
                b.v_cache[blk, :, slot] = nan
                if b.kv_dtype == "fp8" and not seen[t // 16 * 16:t // 16 * 16 + 16].any():
                    b.k_scale[blk] = b.v_scale[blk] = np.nan
    shape, kv, q, bids = rt.upload_batch(b)
    for split in (0, 64):
        att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, kv_split_tokens=split,
                                row_first=first, row_end=end)
        got = rt.to_host_f64(att.run(q, softcap=20.0, slopes=torch.from_numpy(slopes).cuda()))
        torch.cuda.synchronize()
        within(got, want, bound, f"{layer} {mask} split {split}")
