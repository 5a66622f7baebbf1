"""The 4-bit cache on the GPU, through the C ABI: its append bit for bit, its
attention (decode rows of every group size, prefill tiles, splits), its rows
read back, parked and resumed, and a step of all of them together; and the rows
read back from the other cache formats."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import synth  # noqa: E402
from oracle import attention as oa  # noqa: E402
from oracle import codecs, kvappend  # noqa: E402
from synth.attn_inputs import make_batch_from_lengths, round_to_bf16_bits  # noqa: E402
from tests.attn_bound import reference, within  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _batch(q_lens, ctx_lens, hq=32, hkv=8, kv="fp4", d=128, seed=0, spare=8, **kw):
    io = "f32" if kv == "f32" else "bf16"
    pool = sum(-(-c // 16) for c in ctx_lens) + spare
    return make_batch_from_lengths("fp4", q_lens, ctx_lens, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, q_dtype=io,
                                   kv_dtype=kv, out_dtype=io, n_pool_blocks=pool, seed=seed, **kw)


def _same(got, want, what):
    got = got.contiguous().view(torch.uint8).cpu().numpy().reshape(-1)
    want = np.ascontiguousarray(want).view(np.uint8).reshape(-1)
    bad = np.count_nonzero(got != want)
    assert got.size == want.size and bad == 0, f"{what}: {bad} of {got.size} bytes differ"


def _attend(b, **kw):
    from paper_2512_04013_amd import runtime as rt
    shape, kv, q, bids = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids, **kw)
    out = att.run(q)
    torch.cuda.synchronize()
    return att, rt.to_host_f64(out)


HEADS = [(8, 8), (16, 8), (32, 8), (64, 8), (3, 3), (8, 1), (1, 1)]


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_decode_rows(hq, hkv):
    ctx = [1, 2, 15, 16, 17, 31, 33, 64, 100, 300, 1111, 2500]
    say(f"[fp4 rows] {hq}/{hkv}")
    b = _batch([1] * len(ctx), ctx, hq, hkv, seed=hq)
    want, bound = reference(b)
    for split in (0, 32, 16):
        att, got = _attend(b, kv_split_tokens=split)
        assert att.info.num_prefill_items == 0
        within(got, want, bound, f"{hq}/{hkv} split {split}")


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_prefill_tiles_beside_decodes(hq, hkv):
    q = [2, 1, 33, 64, 1, 129, 20]
    ctx = [2, 700, 50, 64, 5, 400, 300]
    say(f"[fp4 tiles] {hq}/{hkv}")
    b = _batch(q, ctx, hq, hkv, seed=hq + 1)
    want, bound = reference(b)
    for split in (0, 64):
        att, got = _attend(b, kv_split_tokens=split)
        assert att.info.num_prefill_items > 0
        within(got, want, bound, f"{hq}/{hkv} split {split}")


def test_long_tiles_are_split_and_merged():
    say("[fp4 long tiles]")
    b = _batch([40], [9000], 8, 1, seed=5)
    att, got = _attend(b)
    assert att.info.num_tile_merge_groups > 0
    want, bound = reference(b)
    within(got, want, bound, "split tiles")


@pytest.mark.parametrize("std", [6.0, 40.0])
def test_sharp_scores(std):
    say(f"[fp4 sharp] {std}")
    b = _batch([1, 1, 40, 1], [500, 40, 90, 2000], seed=9, q_std=std)
    want, bound = reference(b)
    within(_attend(b)[1], want, bound, f"std {std}")


def test_keys_and_queries_of_very_different_sizes():
    """Queries keep every bit that counts beside large elements of the same
    vector, keys and values have the range of their scales."""
    b = _batch([1, 1, 30], [100, 33, 64], 16, 4, seed=11)
    rng = np.random.default_rng(2)
    spread = np.exp2(rng.integers(-12, 1, b.q.shape)).astype(np.float32)
    b.q = round_to_bf16_bits(codecs.bf16_bits_to_f64(b.q).astype(np.float32) * spread)
    h = b.num_kv_heads
    for cache, up in ((b.k_cache, 3), (b.v_cache, 40)):
        live = cache[:, h * 1024:]
        live[live != 255] += np.uint8(up)
    want, bound = reference(b)
    within(_attend(b)[1], want, bound, "spread")
    b.q = np.zeros_like(b.q)
    want, bound = reference(b)
    within(_attend(b)[1], want, bound, "zero queries")


CASES = [([20, 1, 1, 33, 1, 7], [25, 17, 16, 70, 1, 7], 8, 8), ([1, 70, 1, 3, 128], [200, 70, 1000, 29, 700], 32, 8),
         ([5, 1], [5, 2], 3, 3), ([16, 32, 1], [16, 48, 33], 64, 8)]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("std", [1.0, 0.0, 1e-30, 1e30])
def test_append_is_bit_exact(case, std):
    from paper_2512_04013_amd import runtime as rt
    q, ctx, hq, hkv = CASES[case]
    say(f"[fp4 append] case {case} std {std}")
    b = synth.poison_new_slots(_batch(q, ctx, hq, hkv, seed=case))
    k_new, v_new = synth.make_new_kv(b, seed=50 + case, std=std)
    k_new[0, 0, :7] = [0x3E80, 0x3F40, 0x8000, 0x3FA0, 0x40A0, 0x40DC, 0xBE80]   # 0.25, 0.75, -0, 1.25, 5, 6.9, -0.25
    shape, kv, qd, bids = rt.upload_batch(b)
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, b.block_ids, bids)
    att.append(rt.to_device_array(k_new, "bf16", "cuda"), rt.to_device_array(v_new, "bf16", "cuda"))
    torch.cuda.synchronize()
    k, v, _, _ = kvappend.append(b.k_cache, b.v_cache, None, None, "fp4", k_new, v_new, b.q_start, b.ctx_len,
                                 b.bt_start, b.block_ids)
    _same(kv.k_cache, k, "k")
    _same(kv.v_cache, v, "v")
    if std == 1.0:
        got = rt.to_host_f64(att.run(qd))
        want, bound = reference(b, k_cache=k, v_cache=v)
        within(got, want, bound, f"attention after append, case {case}")


@pytest.mark.parametrize("kv_dtype,d", [("fp4", 128), ("fp8", 128), ("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_rows_read_back(kv_dtype, d):
    from paper_2512_04013_amd import runtime as rt
    say(f"[read] {kv_dtype} {d}")
    b = _batch([1, 1, 1], [37, 16, 5], 6, 3, kv=kv_dtype, d=d, seed=4)
    shape, kv, _, _ = rt.upload_batch(b)
    order = np.random.default_rng(0).permutation(37)
    order = np.concatenate([order, order[:3]])                        # any order, some twice
    ids = b.blocks_of(0).astype(np.int64)
    slots = ids[order // 16] * 16 + order % 16
    far = np.array([-1, b.num_pool_blocks * 16, -(1 << 62), (1 << 62)], np.int64)
    k, v = kv.read(torch.from_numpy(np.concatenate([slots, far])).cuda())
    torch.cuda.synchronize()
    for got, cache, scale, is_v in ((k, b.k_cache, b.k_scale, False), (v, b.v_cache, b.v_scale, True)):
        want = oa.materialise_kv(cache, scale, kv_dtype, b.blocks_of(0), 37, is_v=is_v)[order]
        got = rt.to_host_f64(got)
        assert not got[len(order):].any(), "slots outside the pool read as zero"
        if kv_dtype == "fp8":        # code * scale, rounded once to fp32 and once to bf16
            assert (np.abs(got[:len(order)] - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want)).all()
        else:
            assert (got[:len(order)] == want).all()
    k, v = kv.read(torch.empty(0, dtype=torch.int64, device="cuda"))
    assert k.shape == v.shape == (0, 3, d)


def test_large_slots_pass_32_bits():
    """Rows beyond 4 GiB of a pool: the same bytes as read through torch."""
    from paper_2512_04013_amd import make_shape
    from paper_2512_04013_amd import runtime as rt
    shape = make_shape(8, 8, 128, "bf16", "fp4", "bf16", 0.1)
    blocks = (5 << 30) // (8 * 1088)
    pool = torch.zeros(blocks, 8 * 1088, dtype=torch.uint8, device="cuda")
    last = torch.randint(0, 250, (4, 8 * 1088), dtype=torch.uint8, device="cuda")
    last[:, 8 * 1024:] = 127
    pool[-4:] = last
    kv = rt.PagedKV(shape, pool, pool, staging_bytes=1)
    slots = torch.arange((blocks - 4) * 16, blocks * 16, device="cuda")
    k, v = kv.read(slots)
    small = rt.PagedKV(shape, last, last, staging_bytes=1)
    k2, v2 = small.read(torch.arange(64, device="cuda"))
    assert torch.equal(k, k2) and torch.equal(v, v2) and k.abs().sum() > 0
    bids = torch.arange(blocks - 4, blocks, dtype=torch.int32, device="cuda")
    low = torch.arange(4, dtype=torch.int32, device="cuda")
    outs = []
    q = torch.randn(34, 8, 128, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    for p, first in ((kv, blocks - 4), (small, 0)):
        ids = np.array([0, 1, 2, 3, 0], np.int32) + first            # a decode row and a chunk
        att = rt.MixedAttention(shape, p, [0, 1, 34], [30, 33], [0, 2, 5], ids, torch.from_numpy(ids).cuda(), check_blocks=False)
        outs.append(att.run(q).clone())
    assert torch.equal(*outs)


def test_blocks_outside_the_pool_count_for_nothing():
    from paper_2512_04013_amd import runtime as rt
    say("[fp4 bad blocks]")
    b = _batch([1, 40], [100, 90], 32, 8, seed=21)
    shape, kv, q, _ = rt.upload_batch(b)
    bad = b.block_ids.copy()
    bad[2], bad[9] = -5, b.num_pool_blocks + 7
    att = rt.MixedAttention(shape, kv, b.q_start, b.ctx_len, b.bt_start, None, torch.from_numpy(bad).cuda(),
                            check_blocks=False)
    got = rt.to_host_f64(att.run(q))
    torch.cuda.synchronize()
    # the decode row: its third block's keys are left out
    k = oa.materialise_kv(b.k_cache, None, "fp4", b.blocks_of(0), 100)
    v = oa.materialise_kv(b.v_cache, None, "fp4", b.blocks_of(0), 100, is_v=True)
    keep = np.r_[0:32, 48:100]
    want = oa.attend_request(codecs.bf16_bits_to_f64(b.q[:1]), k[keep], v[keep], 32, 8, b.softmax_scale)
    assert np.isfinite(got).all() and np.abs(got[:1] - want).max() <= 2.0 ** -6 * np.abs(v).max()


def test_park_and_resume_move_the_bytes():
    from paper_2512_04013_amd import runtime as rt
    b = _batch([1, 1], [50, 33], 6, 3, seed=6, spare=12)
    shape, kv, q, bids = rt.upload_batch(b)
    assert kv.record_bytes == 2 * 3 * 1088
    before = kv.k_cache.clone(), kv.v_cache.clone()
    src = b.block_ids
    dst = np.setdiff1d(np.arange(b.num_pool_blocks), src)[:len(src)].astype(np.int32)
    host = kv.host_buffer(len(src))
    kv.park(src, torch.from_numpy(src).cuda(), host)
    torch.cuda.synchronize()
    kv.k_cache[torch.from_numpy(src.astype(np.int64)).cuda()] = 255
    kv.resume(dst, torch.from_numpy(dst).cuda(), host)
    torch.cuda.synchronize()
    for now, was in zip((kv.k_cache, kv.v_cache), before):
        assert torch.equal(now[torch.from_numpy(dst.astype(np.int64)).cuda()], was[torch.from_numpy(src.astype(np.int64)).cuda()])


def test_a_request_moves_from_fp8_to_four_bits_and_goes_on():
    """Read out of an fp8 pool, appended to a 4-bit pool, then a decode step with
    its append, captured in a graph and replayed: every replay equals the eager
    result and float64."""
    from paper_2512_04013_amd import runtime as rt
    say("[fp4 flow]")
    old = _batch([1], [200], 32, 8, kv="fp8", seed=31)
    shape8, kv8, _, _ = rt.upload_batch(old)
    pos = np.arange(200)
    slots = old.blocks_of(0).astype(np.int64)[pos // 16] * 16 + pos % 16
    k_rows, v_rows = kv8.read(torch.from_numpy(slots).cuda())
    step = _batch([1], [201], 32, 8, seed=32)
    shape, kv, q, bids = rt.upload_batch(synth.poison_new_slots(step))
    kv.k_cache.fill_(255)
    kv.v_cache.fill_(255)
    move = rt.MixedAttention(shape, kv, [0, 200], [200], step.bt_start, step.block_ids, bids)
    move.append(k_rows, v_rows)
    k_new, v_new = synth.make_new_kv(step, seed=33)
    kd, vd = rt.to_device_array(k_new, "bf16", "cuda"), rt.to_device_array(v_new, "bf16", "cuda")
    att = rt.MixedAttention(shape, kv, step.q_start, step.ctx_len, step.bt_start, step.block_ids, bids, kv_split_tokens=64)
    att.append(kd, vd)
    eager = att.run(q).clone()
    torch.cuda.synchronize()
    rows = [np.concatenate([r.view(torch.int16).cpu().numpy().view(np.uint16), n])
            for r, n in ((k_rows, k_new), (v_rows, v_new))]
    empty = np.full_like(step.k_cache, 255)
    k, v, _, _ = kvappend.append(empty, empty, None, None, "fp4", rows[0], rows[1], [0, 201], [201], step.bt_start, step.block_ids)
    _same(kv.k_cache, k, "k")
    _same(kv.v_cache, v, "v")
    want, bound = reference(step, k_cache=k, v_cache=v)
    within(rt.to_host_f64(eager), want, bound, "decode after the move")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            att.append(kd, vd)
            att.run(q)
    for _ in range(3):
        att.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(att.out, eager)
