"""Block ids outside the pool, in tables that no host check has seen: their keys
count for nothing in decode rows, prefill rows and tiles of every cache format,
whole and split, plain and with modified scores; a row that is left without keys
gives zeros; nothing outside the pool is read.

The bound is that of attn_bound.py, on the weights of the keys that remain; the
fp8 tile products add theirs: queries rounded to E4M3 (taken as they are then),
and probabilities of the FP8 form by 2^-4 of each, gone below 2^-15 of the row's
largest."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402
from oracle.codecs import storage_to_f64  # noqa: E402
from synth.attn_inputs import make_batch_from_lengths  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

Q = [1, 40, 1, 129, 5, 1, 20]
CTX = [100, 90, 20, 400, 30, 16, 20]
#       request: blocks of its table that lie outside the pool (the last two have no other)
HOLES = {0: [2], 1: [0, 5], 2: [1], 3: [3, 4, 5, 6, 9, 24], 4: [0], 5: [0], 6: [0, 1]}


def _batch(layer, seed):
    hq, hkv, d, kv = layer
    io = "f32" if kv == "f32" else "bf16"
    return make_batch_from_lengths("bad", Q, CTX, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q_dtype=io, kv_dtype=kv,
                                   out_dtype=io, n_pool_blocks=sum(-(-c // 16) for c in CTX) + 4, seed=seed, q_std=2.0)


def _table(b):
    ids = b.block_ids.copy()
    for i, (r, blocks) in enumerate(HOLES.items()):
        for k in blocks:
            ids[int(b.bt_start[r]) + k] = [-1, b.num_pool_blocks, -2 ** 31, 2 ** 31 - 1][(i + k) % 4]
    return ids


def _reference(b, softcap, slopes, tile_path):
    out = np.zeros((b.total_q, b.num_q_heads, b.head_dim))
    bound = np.full_like(out, 1e-30)
    g = b.num_q_heads // b.num_kv_heads
    fine = b.kv_dtype == "f32"
    for r in range(b.num_reqs):
        q0, q1, ctx = int(b.q_start[r]), int(b.q_start[r + 1]), int(b.ctx_len[r])
        keep = np.ones(ctx)
        for k in HOLES[r]:
            keep[16 * k:16 * k + 16] = 0
        k, v = (oa.materialise_kv(c, s, b.kv_dtype, b.blocks_of(r), ctx, is_v=is_v)
                for c, s, is_v in ((b.k_cache, b.k_scale, False), (b.v_cache, b.v_scale, True)))
        q = storage_to_f64(b.q[q0:q1], b.q_dtype)
        fp8 = tile_path > 1 and q1 - q0 > 1
        if fp8:
            q = oa.round_query_rows_e4m3(q)
        for h in range(b.num_q_heads):
            p = oa.request_weights(q, k, h, b.num_q_heads, b.num_kv_heads, b.softmax_scale, softcap, slopes) * keep
            total = p.sum(1, keepdims=True)
            p /= np.where(total > 0, total, 1.0)
            vh = v[:, h // g]
            o = p @ vh
            size = (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max(1) * b.softmax_scale
            away = 0.0 if slopes is None else abs(float(slopes[h])) * ctx
            d = 2.0 ** -24 * (b.head_dim * size + 32 * (1 + size + away) + ctx) + softcap * 2.0 ** -20
            rel = d + (0.0 if fine else 2.0 ** -8) + (2.0 ** -4 if fp8 and tile_path == 3 else 0.0)
            out[q0:q1, h] = o
            bound[q0:q1, h] += (1.01 * rel)[:, None] * (p @ np.abs(vh) + np.abs(o)) + (2.0 ** -24 if fine else 2.0 ** -8) * np.abs(o)
            if fp8 and tile_path == 3:
                bound[q0:q1, h] += (ctx * 2.0 ** -15 * p.max(1))[:, None] * (np.abs(vh).max(0) + np.abs(o))
    return out, bound


LAYERS = {"f32-8x2-d64": (8, 2, 64, "f32"), "bf16-4x4-d64": (4, 4, 64, "bf16"), "bf16-8x2-d128": (8, 2, 128, "bf16"),
          "bf16-8x1-d128": (8, 1, 128, "bf16"), "fp8-2x2-d128": (2, 2, 128, "fp8"), "fp8-16x2-d128": (16, 2, 128, "fp8"),
          "fp4-4x2-d128": (4, 2, 128, "fp4"), "fp4-8x1-d128": (8, 1, 128, "fp4")}
PLAIN = [(name, 1, False) for name in LAYERS]
SCORED = [(name, 1, True) for name in LAYERS]
FP8 = [("fp8-2x2-d128", 2, False), ("fp8-16x2-d128", 2, False), ("fp8-2x2-d128", 3, False), ("fp8-16x2-d128", 3, False)]


@pytest.mark.parametrize("name,tile_path,scored", PLAIN + SCORED + FP8)
@pytest.mark.parametrize("split", [0, 32])
def test_keys_outside_the_pool_count_for_nothing(name, tile_path, scored, split):
    from paper_2512_04013_amd import runtime as rt
    say(f"[bad blocks] {name} tiles {tile_path} scored {scored} split {split}")
    b = _batch(LAYERS[name], seed=7)
    cap, slopes = (20.0, np.linspace(-0.05, 0.2, b.num_q_heads).astype(np.float32)) if scored else (0.0, None)
    want, bound = _reference(b, cap, slopes, tile_path)
    shape, kv, q, _ = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, None, torch.from_numpy(_table(b)).cuda(),
                            check_blocks=False, kv_split_tokens=split, tile_path=tile_path)
    att.out.fill_(float("nan"))
    got = rt.to_host_f64(att.run(q, softcap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda()))
    torch.cuda.synchronize()
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / bound).max()
    say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0
    for r in (5, 6):
        assert not got[int(b.q_start[r]):int(b.q_start[r + 1])].any(), "a row without keys gives zeros"
    first = int(b.q_start[4])                      # rows 0 .. 3 of request 4 are at positions 25 ..: block 1 is theirs
    assert got[first:first + 5].any()


@pytest.mark.parametrize("layer", ["bf16-8x1-d128", "fp8-16x2-d128", "fp4-8x1-d128", "bf16-4x4-d64"])
def test_split_tiles_with_whole_spans_outside_the_pool(layer):
    """A long chunk whose tiles are split over spans, one of them without a single
    usable block."""
    from paper_2512_04013_amd import runtime as rt
    hq, hkv, d, kvd = LAYERS[layer]
    say(f"[bad spans] {layer}")
    ctx = 9000
    b = make_batch_from_lengths("bad", [40], [ctx], num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q_dtype="bf16", kv_dtype=kvd,
                                out_dtype="bf16", n_pool_blocks=570, seed=3)
    shape, kv, q, _ = rt.upload_batch(b)
    ids = b.block_ids.copy()
    ids[:400] = -7
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, None, torch.from_numpy(ids).cuda(), check_blocks=False)
    assert att.info.num_tile_merge_groups > 0
    got = rt.to_host_f64(att.run(q))
    # the same rows over the 2600 keys that remain
    short = rt.MixedAttention(shape, kv, [0, 40], [ctx - 6400], [0, 163], b.block_ids[400:563],
                              torch.from_numpy(b.block_ids[400:].copy()).cuda())
    want = rt.to_host_f64(short.run(q))
    v = np.abs(oa.materialise_kv(b.v_cache, b.v_scale, kvd, b.blocks_of(0), ctx, is_v=True)[6400:]).max()
    # both sides: bf16 weights (2^-8 each, sums of a few hundred keys) and one output rounding
    assert np.isfinite(got).all() and np.abs(got - want).max() <= 2 * 2.0 ** -8 * (v + np.abs(want).max())
