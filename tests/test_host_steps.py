"""Steps whose lengths are on the GPU, as far as the CPU goes: angles of rotary
positions, and every call that is refused before anything is launched."""

import ctypes as C
import math

import numpy as np
import pytest

import paper_2512_04013_amd as aug
from oracle import rope as orope

ROPES = [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0),
         dict(base=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original_len=8192),
         dict(base=1e6, scaling="ramp", factor=4.0, low=1.0, high=32.0, original_len=32768),
         dict(scaling="ramp", factor=40.0, low=1.0, high=32.0, original_len=64)]


@pytest.mark.parametrize("dim", [16, 48, 64, 128])
@pytest.mark.parametrize("kw", ROPES)
def test_angles(dim, kw):
    rope = aug.aug_rope_init(dim, **kw)
    want = orope.frequencies(dim, **kw) / (2 * math.pi)
    got = np.array(list(rope.turns))
    # a power, two products and two quotients, each correct to a unit or two in the last place
    np.testing.assert_allclose(got[:dim // 2], want, rtol=16 * 2.0 ** -53)
    assert (got[dim // 2:] == 0).all() and rope.rotary_dim == dim


@pytest.mark.parametrize("kw,status", [
    (dict(rotary_dim=0), aug.AUG_ERR_UNSUPPORTED), (dict(rotary_dim=24), aug.AUG_ERR_UNSUPPORTED),
    (dict(rotary_dim=144), aug.AUG_ERR_UNSUPPORTED), (dict(rotary_dim=-16), aug.AUG_ERR_UNSUPPORTED),
    (dict(base=1.0), aug.AUG_ERR_INVALID), (dict(base=float("nan")), aug.AUG_ERR_INVALID), (dict(base=float("inf")), aug.AUG_ERR_INVALID),
    (dict(scaling=4), aug.AUG_ERR_INVALID), (dict(scaling=-1), aug.AUG_ERR_INVALID),
    (dict(scaling="linear", factor=0.0), aug.AUG_ERR_INVALID), (dict(scaling="linear", factor=float("nan")), aug.AUG_ERR_INVALID),
    (dict(scaling="linear", factor=1e-5), aug.AUG_ERR_INVALID),
    (dict(scaling="bands", factor=2.0), aug.AUG_ERR_INVALID),
    (dict(scaling="bands", factor=2.0, original_len=10, low=4.0, high=4.0), aug.AUG_ERR_INVALID),
    (dict(scaling="ramp", factor=2.0, original_len=10, low=0.0, high=4.0), aug.AUG_ERR_INVALID),
    (dict(scaling="ramp", factor=2.0, original_len=10, low=1.0, high=float("inf")), aug.AUG_ERR_INVALID),
    (dict(magnitude=float("nan")), aug.AUG_ERR_INVALID), (dict(magnitude=float("inf")), aug.AUG_ERR_INVALID)])
def test_angles_refused(kw, status):
    with pytest.raises(aug.AugError) as e:
        aug.aug_rope_init(**{"rotary_dim": 64, **kw})
    assert e.value.status == status


def test_angles_refuse_null_and_flags():
    p, r = aug.aug_rope_params(64, 2, 0, 0, 10000.0, 1.0, 1.0, 2.0, 1.0), aug.aug_rope()
    assert aug.lib().aug_rope_init(C.byref(p), C.byref(r)) == aug.AUG_ERR_INVALID
    p.interleaved = 1
    assert aug.lib().aug_rope_init(None, C.byref(r)) == aug.AUG_ERR_INVALID
    assert aug.lib().aug_rope_init(C.byref(p), None) == aug.AUG_ERR_INVALID
    assert aug.lib().aug_rope_init(C.byref(p), C.byref(r)) == aug.AUG_OK


# ---- device calls: addresses that are never used, since every call is refused -------------

P = 1 << 20          # an aligned address


def _tables(**kw):
    f = dict(num_reqs=4, max_rows=8, max_blocks=4, num_pool_blocks=16, max_draft=4, reserved=0)
    f.update({n: P for n, _ in aug.aug_step_tables_args._fields_[6:]})
    f.update(kw)
    return aug.aug_step_tables_args(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(num_reqs=-1), aug.AUG_ERR_INVALID), (dict(max_rows=-1), aug.AUG_ERR_INVALID), (dict(max_rows=2 ** 31 - 1), aug.AUG_ERR_INVALID),
    (dict(max_blocks=0), aug.AUG_ERR_INVALID), (dict(num_pool_blocks=0), aug.AUG_ERR_INVALID), (dict(max_draft=-1), aug.AUG_ERR_INVALID),
    (dict(max_draft=65), aug.AUG_ERR_INVALID), (dict(reserved=1), aug.AUG_ERR_INVALID), (dict(num_reqs=4097), aug.AUG_ERR_UNSUPPORTED),
    (dict(max_blocks=(1 << 20) + 1), aug.AUG_ERR_UNSUPPORTED), (dict(max_draft=0), aug.AUG_ERR_INVALID),
    (dict(max_draft=0, parents=None), aug.AUG_ERR_INVALID), (dict(max_draft=0, seen=None), aug.AUG_ERR_INVALID)]
    + [({n: None}, aug.AUG_ERR_INVALID) for n, _ in aug.aug_step_tables_args._fields_[6:] if n != "parents"])
def test_tables_refused(kw, status):
    a = _tables(**kw)
    assert aug.lib().aug_step_tables(C.byref(a), None) == status, aug.aug_last_error()
    assert aug.aug_last_error()


def test_tables_of_nothing():
    assert aug.lib().aug_step_tables(None, None) == aug.AUG_ERR_INVALID
    a = aug.aug_step_tables_args(0, 0, 1, 1, 4, 0)
    assert aug.lib().aug_step_tables(C.byref(a), None) == aug.AUG_OK


def _shape(kv="bf16", hq=8, hkv=2, d=128):
    io = "f32" if kv == "f32" else "bf16"
    return aug.make_shape(hq, hkv, d, io, kv, io, 0.1)


def _rows(shape=None, rope=None, **kw):
    a = dict(positions=P, rows=3, q=P, q_stride=1024, k=P, k_stride=256, q_out=P, q_out_stride=1024, k_out=P, k_out_stride=256)
    a.update(kw)
    rope = aug.aug_rope_init(64) if rope is None else rope
    return aug.lib().aug_rope_rows(C.byref(shape or _shape()), C.byref(rope), *a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(positions=None), dict(rows=-1), dict(q_out=None), dict(q=None), dict(k_out=None), dict(k=None),
    dict(q=None, q_out=None, k=None, k_out=None), dict(q=P + 8), dict(k=P + 2), dict(q_out=P + 4, q=P + 4), dict(q_stride=1016, q_out_stride=1016),
    dict(q_stride=1028), dict(k_stride=-256), dict(k_out_stride=0), dict(q_out_stride=2048), dict(k_stride=1 << 50)])
def test_rows_refused(kw):
    assert _rows(**kw) == aug.AUG_ERR_INVALID and aug.aug_last_error()


def test_rows_shapes_refused():
    assert _rows(rows=0) == aug.AUG_OK
    assert aug.lib().aug_rope_rows(C.byref(_shape()), None, P, 1, P, 1024, None, 0, P, 1024, None, 0, None) == aug.AUG_ERR_INVALID
    assert _rows(shape=_shape(hq=7)) == aug.AUG_ERR_INVALID
    assert _rows(shape=_shape(d=64), rope=aug.aug_rope_init(128)) == aug.AUG_ERR_UNSUPPORTED
    for name, value in (("rotary_dim", 24), ("rotary_dim", 0), ("interleaved", 2), ("reserved", 1)):
        rope = aug.aug_rope_init(64)
        setattr(rope, name, value)
        assert _rows(rope=rope) == aug.AUG_ERR_INVALID


def _append(shape=None, rope=True, **kw):
    a = dict(positions=P, slots=P, rows=3, live_rows=None, q=P, q_stride=1024, k=P, k_stride=256, v=P, v_stride=256, q_out=P,
             q_out_stride=1024, k_cache=P, v_cache=P, k_scale=P, v_scale=P, num_pool_blocks=4)
    a.update(kw)
    r = C.byref(aug.aug_rope_init(64)) if rope else None
    return aug.lib().aug_rope_append(C.byref(shape or _shape()), r, *a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(positions=None), dict(slots=None), dict(slots=P + 4), dict(rows=-1), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None),
    dict(k_cache=None), dict(v_cache=None), dict(k_cache=P + 8), dict(num_pool_blocks=0), dict(k=P + 8), dict(v_stride=128),
    dict(v_stride=260), dict(q_out_stride=2048), dict(rope=False), dict(rope=False, positions=None),
    dict(rope=False, q=None, q_out=None), dict(live_rows=P + 2)])
def test_append_refused(kw):
    assert _append(**kw) == aug.AUG_ERR_INVALID and aug.aug_last_error()


def test_append_shapes_refused():
    assert _append(rows=0) == aug.AUG_OK
    assert _append(shape=_shape("fp8"), k_scale=None) == aug.AUG_ERR_INVALID
    assert _append(shape=_shape("fp8"), v_scale=None) == aug.AUG_ERR_INVALID
    assert _append(shape=_shape("fp4", d=64)) == aug.AUG_ERR_UNSUPPORTED
    assert _append(shape=_shape(hq=6)) == aug.AUG_ERR_UNSUPPORTED


def test_python_refuses():
    torch = pytest.importorskip("torch")
    from paper_2512_04013_amd import runtime as rt
    pool = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    kv = rt.PagedKV(_shape(), pool, pool.clone(), staging_bytes=1)
    slots, rows = torch.zeros(3, dtype=torch.int64), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    q, pos = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    rope = rt.Rope(64)
    bad = [dict(slots=slots.int()), dict(slots=slots[:2]), dict(k=rows.float()), dict(v=rows[:, :1]), dict(k=rows.transpose(0, 1)),
           dict(k=torch.zeros(3, 128, 2, dtype=torch.bfloat16).transpose(1, 2)), dict(q=q), dict(positions=pos), dict(rope=rope),
           dict(q=q, rope=rope, positions=pos.long()), dict(q=q[:, :4], rope=rope, positions=pos),
           dict(q_out=q, rope=rope, positions=pos), dict(q=q, q_out=q.float(), rope=rope, positions=pos),
           dict(live_rows=slots[:1]), dict(live_rows=pos)]
    for kw in bad:
        with pytest.raises(ValueError):
            kv.append_rows(**{"slots": slots, "k": rows, "v": rows, **kw})
    for kw in (dict(q=q.float()), dict(k=rows[:2]), dict(q=q, k_out=rows), dict(q=q, q_out=q[:2])):
        with pytest.raises(ValueError):
            rt.rope_rows(_shape(), rope, pos, **kw)
    with pytest.raises(ValueError):
        rt.rope_rows(_shape(), rope, pos.long(), q)
    table, held = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    free = torch.arange(8, dtype=torch.int32)
    for kw in (dict(block_table=table), dict(block_table=table, held=held), dict(block_table=table[:1], held=held, free_ids=free),
               dict(block_table=table, held=held.long(), free_ids=free), dict(free_ids=free[:4]), dict(free_count=9)):
        with pytest.raises(ValueError):
            rt.StepTables(2, 8, 4, 8, device="cpu", **kw)
    t = rt.StepTables(2, 8, 4, 8, device="cpu", block_table=table, held=held, free_ids=free)
    two = torch.zeros(2, dtype=torch.int32)
    for args in ((two[:1], two), (two, two.long()), (two, two, two), (two.repeat(2)[::2], two)):
        with pytest.raises(ValueError):
            t.update(*args)


# ---- attention of drafts ---------------------------------------------------------------------

def _batch(**kw):
    f = dict(num_reqs=4, max_rows=32, max_blocks=17, max_draft=8, q_start=P, kv_len=P, block_table=P, seen=P)
    f.update(kw)
    return aug.aug_tree_batch(**f)


def test_tree_sizes():
    """Room for any lengths: the items of every request in one span (128 columns each at most) and those of the splits;
    partials of 2048 split items of 32, 64 or 128 columns; nothing of these for tables of 128 keys, or of 256 and
    up to 32 columns."""
    for draft, hq, kv, tiles, columns in ((1, 8, "bf16", 1, 32), (8, 8, "bf16", 1, 32), (9, 8, "bf16", 1, 64), (17, 8, "f32", 1, 128),
                                          (64, 8, "bf16", 2, 128), (64, 16, "bf16", 4, 128)):
        shape = _shape(kv, hq=hq)
        plan, workspace = aug.aug_tree_plan_size(shape, _batch(max_draft=draft))
        whole = 4 * 2 * tiles
        assert plan == 64 + 32 * (1024 + whole) + 32 * whole
        assert workspace == 16 + (1024 + whole) * columns * 130 * 4
        for blocks, split in ((1, False), (8, False), (9, columns > 32), (16, columns > 32)):
            got = aug.aug_tree_plan_size(shape, _batch(max_draft=draft, max_blocks=blocks))
            assert got == ((plan, workspace) if split else (64 + 32 * (1024 + whole), 16)), blocks
    plan, workspace = aug.aug_tree_plan_size(_shape(), _batch(num_reqs=4096, max_draft=1))
    assert plan == 64 + 32 * (1024 + 8192) + 32 * 1024 and workspace == 16 + 2048 * 32 * 130 * 4


@pytest.mark.parametrize("kw,status", [
    (dict(num_reqs=-1), aug.AUG_ERR_INVALID), (dict(max_rows=-1), aug.AUG_ERR_INVALID), (dict(max_blocks=0), aug.AUG_ERR_INVALID),
    (dict(max_draft=0), aug.AUG_ERR_INVALID), (dict(max_draft=65), aug.AUG_ERR_INVALID), (dict(num_reqs=4097), aug.AUG_ERR_UNSUPPORTED),
    (dict(max_blocks=(1 << 20) + 1), aug.AUG_ERR_UNSUPPORTED)])
def test_tree_batches_refused(kw, status):
    s, b, n = _shape(), _batch(**kw), C.c_size_t()
    L = aug.lib()
    assert L.aug_tree_plan_size(C.byref(s), C.byref(b), C.byref(n), C.byref(n)) == status
    assert L.aug_tree_plan(C.byref(s), C.byref(b), P, 1 << 40, None) == status
    assert L.aug_attn_tree(C.byref(s), C.byref(b), P, P, P, P, P, P, 4, P, P, 1 << 40, None) == status


def test_tree_calls_refused():
    L, s, n = aug.lib(), _shape(), C.c_size_t()
    b = _batch()
    assert L.aug_tree_plan_size(C.byref(s), None, C.byref(n), C.byref(n)) == aug.AUG_ERR_INVALID
    assert L.aug_tree_plan_size(C.byref(s), C.byref(b), None, C.byref(n)) == aug.AUG_ERR_INVALID
    assert L.aug_tree_plan_size(None, C.byref(b), C.byref(n), C.byref(n)) == aug.AUG_ERR_INVALID
    many = _batch(num_reqs=4096, max_draft=64)
    assert L.aug_tree_plan_size(C.byref(_shape(hq=8192, hkv=1024)), C.byref(many), C.byref(n), C.byref(n)) == aug.AUG_ERR_UNSUPPORTED
    plan = lambda **kw: L.aug_tree_plan(C.byref(s), C.byref(_batch(**{k: v for k, v in kw.items() if k in ("q_start", "kv_len")})),  # noqa: E731
                                        kw.get("plan", P), kw.get("size", 1 << 40), None)
    for kw in (dict(q_start=None), dict(kv_len=None), dict(plan=None), dict(plan=P + 8)):
        assert plan(**kw) == aug.AUG_ERR_INVALID
    assert plan(size=100) == aug.AUG_ERR_NO_SPACE

    def attend(shape=s, **kw):
        batch = _batch(**{k: kw.pop(k) for k in ("block_table", "seen", "num_reqs", "max_rows") if k in kw})
        a = dict(plan=P, q=P, k=P, v=P, ks=P, vs=P, pool=4, out=P, workspace=P, size=1 << 40)
        a.update(kw)
        return L.aug_attn_tree(C.byref(shape), C.byref(batch), *a.values(), None)

    for kw in (dict(plan=None), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(block_table=None), dict(seen=None),
               dict(pool=0), dict(plan=P + 4), dict(q=P + 8), dict(k=P + 8), dict(v=P + 2), dict(out=P + 8), dict(workspace=P + 8)):
        assert attend(**kw) == aug.AUG_ERR_INVALID, kw
    for kw in (dict(workspace=None), dict(size=1000)):
        assert attend(**kw) == aug.AUG_ERR_NO_SPACE, kw
    assert attend(_shape("fp8"), ks=None) == aug.AUG_ERR_INVALID
    assert attend(_shape("fp8"), vs=None) == aug.AUG_ERR_INVALID
    assert attend(num_reqs=0, plan=None) == aug.AUG_OK and attend(max_rows=0, q=None) == aug.AUG_OK


# ---- sampling ------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), aug.AUG_ERR_INVALID), (dict(vocab=0), aug.AUG_ERR_INVALID), (dict(vocab=-5), aug.AUG_ERR_INVALID),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), aug.AUG_ERR_UNSUPPORTED), (dict(dtype=aug.AUG_FP8_E4M3FN), aug.AUG_ERR_INVALID),
    (dict(dtype=-1), aug.AUG_ERR_INVALID), (dict(reserved=1), aug.AUG_ERR_INVALID), (dict(stride=99), aug.AUG_ERR_INVALID),
    (dict(stride=-100), aug.AUG_ERR_INVALID), (dict(stride=1 << 41), aug.AUG_ERR_INVALID), (dict(logits=None), aug.AUG_ERR_INVALID),
    (dict(logits=P + 2), aug.AUG_ERR_INVALID), (dict(logits=P + 1, dtype=aug.AUG_BF16), aug.AUG_ERR_INVALID),
    (dict(uniform=None), aug.AUG_ERR_INVALID), (dict(tokens=None), aug.AUG_ERR_INVALID)])
def test_sample_refused(kw, status):
    f = dict(rows=2, vocab=100, dtype=aug.AUG_F32, reserved=0, stride=100, logits=P, uniform=P, temperature=P, top_k=P, top_p=P, min_p=P,
             tokens=P, probs=P)
    f.update(kw)
    assert aug.lib().aug_sample(C.byref(aug.aug_sample_args(**f)), None) == status and aug.aug_last_error()


def test_sample_of_nothing():
    assert aug.lib().aug_sample(None, None) == aug.AUG_ERR_INVALID
    assert aug.lib().aug_sample(C.byref(aug.aug_sample_args(0, 5, aug.AUG_F32, 0, 5)), None) == aug.AUG_OK


def test_oracle_draws():
    """The oracle itself, where the answer is plain."""
    from oracle import sampling
    x = [0.0, 3.0, 1.0, 3.0]
    assert sampling.draw(x, 0.9, temperature=0.0)[0] == 1 and sampling.draw(x, 0.99, top_k=1)[0] == 1
    assert sampling.draw(x, 0.6, top_k=2)[:2] == (3, 0.5) and sampling.draw(x, 0.4, top_p=0.5)[0] in (1, 3)
    assert sampling.draw(x, 0.99, min_p=0.5)[0] == 3 and sampling.draw([float("nan"), -np.inf], 0.5)[0] == -1
    assert sampling.draw([np.inf, 0.0, np.inf], 0.5)[:2] == (2, 0.5)
