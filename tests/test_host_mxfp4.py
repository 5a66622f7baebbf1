"""CPU tests of the 4-bit cache's entry points: shapes, plans and refusals, all
before any device call."""

import os

import numpy as np
import pytest

import paper_2512_04013_amd as aug
from paper_2512_04013_amd import AugError

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")


def _shape(hq=32, hkv=8, d=128, q="bf16", kv="fp4", out="bf16"):
    return aug.make_shape(hq, hkv, d, q, kv, out, 0.088)


def _plan(shape, q_len=(1, 40), ctx=(700, 300), **kw):
    bt = np.concatenate([[0], np.cumsum([-(-c // 16) for c in ctx])])
    return aug.aug_attn_plan(shape, np.concatenate([[0], np.cumsum(q_len)]), ctx, bt, int(bt[-1]) + 4, **kw)


def test_record_bytes_and_shapes():
    assert aug.aug_kv_record_bytes(_shape()) == 2 * 8 * 1088
    assert aug.aug_kv_record_bytes(_shape(3, 3)) == 2 * 3 * 1088
    for bad in (_shape(d=64), _shape(q="f32"), _shape(out="f32"), _shape(hq=48)):
        assert aug.aug_kv_record_bytes(bad) == 0
        with pytest.raises(AugError) as e:
            _plan(bad)
        assert e.value.status == aug.AUG_ERR_UNSUPPORTED


@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 8), (32, 8), (64, 8)])
def test_rows_run_on_mfma_only(hq, hkv):
    s = _shape(hq, hkv)
    for path in (aug.AUG_ROWS_AUTO, aug.AUG_ROWS_MFMA):
        info, _ = _plan(s, row_path=path)
        assert info.row_path == aug.AUG_ROWS_MFMA and info.tile_path == aug.AUG_TILES_BF16
    with pytest.raises(AugError) as e:
        _plan(s, row_path=aug.AUG_ROWS_VALU)
    assert e.value.status == aug.AUG_ERR_UNSUPPORTED
    for path in (aug.AUG_TILES_FP8_QK, aug.AUG_TILES_FP8):
        with pytest.raises(AugError) as e:
            _plan(s, tile_path=path)
        assert e.value.status == aug.AUG_ERR_UNSUPPORTED
    bad = aug.aug_attn_plan_info.from_buffer_copy(info)
    bad.row_path = aug.AUG_ROWS_VALU
    st = aug.lib().aug_attn_mixed(aug.C.byref(s), aug.C.byref(bad), 16, 16, 16, 16, None, None, 16, 80, 16, 16, 1 << 40, None)
    assert st == aug.AUG_ERR_INVALID and "row path" in aug.aug_last_error()


def test_misaligned_pools_are_refused():
    L, s = aug.lib(), _shape()
    info, _ = _plan(s)
    for k, v in ((24, 16), (16, 20)):
        assert L.aug_attn_mixed(aug.C.byref(s), aug.C.byref(info), 16, 16, k, v, None, None, 16, 80, 16, 16, 1 << 40,
                                None) == aug.AUG_ERR_INVALID
        assert "aligned" in aug.aug_last_error()
        assert L.aug_kv_append(aug.C.byref(s), aug.C.byref(info), 16, 16, 16, k, v, None, None, 16, 80, None) == \
            aug.AUG_ERR_INVALID
        assert "aligned" in aug.aug_last_error()


def test_read_refuses_bad_arguments():
    L, s = aug.lib(), _shape()

    def read(shape=s, k=16, v=16, ks=None, vs=None, slots=16, n=5, pool=9, ko=16, vo=16):
        return L.aug_kv_read(aug.C.byref(shape), k, v, ks, vs, slots, n, pool, ko, vo, None)

    assert read(n=0, k=None, v=None, slots=None, ko=None, vo=None) == aug.AUG_OK
    assert read(n=-1) == read(pool=0) == aug.AUG_ERR_INVALID
    assert L.aug_kv_read(None, 16, 16, None, None, 16, 5, 9, 16, 16, None) == aug.AUG_ERR_INVALID
    for name in ("k", "v", "slots", "ko", "vo"):
        assert read(**{name: None}) == aug.AUG_ERR_INVALID and "NULL" in aug.aug_last_error()
    for name in ("k", "v", "ko", "vo"):
        assert read(**{name: 24}) == aug.AUG_ERR_INVALID and "aligned" in aug.aug_last_error()
    assert read(slots=12) == aug.AUG_ERR_INVALID
    assert read(n=1 << 28) == aug.AUG_ERR_UNSUPPORTED
    assert read(shape=_shape(kv="fp8")) == aug.AUG_ERR_INVALID and "scales" in aug.aug_last_error()
    assert read(shape=_shape(d=96)) == aug.AUG_ERR_UNSUPPORTED


def test_runtime_checks_pools_and_rows():
    torch = pytest.importorskip("torch")
    from paper_2512_04013_amd import runtime as rt
    s = _shape(6, 3)
    pool = torch.zeros(4, 3 * 1088, dtype=torch.uint8)
    kv = rt.PagedKV(s, pool, pool.clone(), staging_bytes=1)
    for bad in (torch.zeros(4, 3 * 1024, dtype=torch.uint8), torch.zeros(4, 3, 16, 64, dtype=torch.uint8),
                torch.zeros(4, 3 * 1088, dtype=torch.int8)):
        with pytest.raises(ValueError):
            rt.PagedKV(s, bad, bad, staging_bytes=1)
        with pytest.raises(ValueError):
            rt.PagedKV(s, pool, bad, staging_bytes=1)
    ok = torch.zeros(3, dtype=torch.int64)
    for slots in (ok.int(), ok.view(1, 3), torch.zeros(6, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            kv.read(slots)
    row = torch.zeros(3, 3, 128, dtype=torch.bfloat16)
    for k in (row.float(), row[:2], torch.zeros(3, 3, 256, dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(ValueError):
            kv.read(ok, k, row)
        with pytest.raises(ValueError):
            kv.read(ok, row, k)
