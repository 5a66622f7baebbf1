"""Tensors in host memory, all of them: the calls that take their device from the tensors refuse
them and launch nothing."""

import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402


def _shape():
    return aug.make_shape(8, 2, 128, "bf16", "bf16", "bf16", 0.1)


def _never(*a, **kw):
    raise AssertionError("launched")


@pytest.fixture(autouse=True)
def nothing_is_launched(monkeypatch):
    from paper_2512_04013_amd import runtime as rt
    for name in ("aug_rope_rows", "aug_rope_append", "aug_step_tables", "aug_tree_plan", "aug_attn_tree", "aug_sample"):
        monkeypatch.setattr(rt, name, _never)


def test_rows():
    from paper_2512_04013_amd import runtime as rt
    pos, q, k = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    for kw in (dict(q=q), dict(k=k), dict(q=q, k=k, q_out=q, k_out=k)):
        with pytest.raises(ValueError, match="host memory"):
            rt.rope_rows(_shape(), rt.Rope(64), pos, **kw)


def test_append():
    from paper_2512_04013_amd import runtime as rt
    pool, rows = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    kv = rt.PagedKV(_shape(), pool, pool.clone(), staging_bytes=1)
    slots, pos = torch.arange(3), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(), dict(rope=rt.Rope(64), positions=pos), dict(live_rows=pos[:1])):
        with pytest.raises(ValueError, match="host memory"):
            kv.append_rows(slots, rows, rows, **kw)


def test_tables_and_drafts():
    from paper_2512_04013_amd import runtime as rt
    t = rt.StepTables(2, 8, 4, 4, device="cpu")
    two = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="host memory"):
        t.update(two, two)
    pool = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    att = rt.TreeAttention(_shape(), rt.PagedKV(_shape(), pool, pool.clone(), staging_bytes=1), t)
    with pytest.raises(ValueError, match="host memory"):
        att.plan()
    att._planned = True
    with pytest.raises(ValueError, match="host memory"):
        att.run(torch.zeros(8, 8, 128, dtype=torch.bfloat16))


def test_logits():
    from paper_2512_04013_amd import runtime as rt
    with pytest.raises(ValueError):
        rt.sample(torch.zeros(2, 9), torch.zeros(2))
