"""How requests pass between tables on the GPU and the calls that take block ids on the host: parked and
resumed under a table, prompts planned on the host over a table's blocks, and tables that take over from others."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
HKV, D, POOL = 2, 128, 40


def _kv(seed=0):
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pools = [torch.randn(POOL, HKV, 16, D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    return rt.PagedKV(aug.make_shape(8, HKV, D, "bf16", "bf16", "bf16", 0.1), *pools)


def _rows(t, kv, r, n):
    """K and V of a request's first n tokens, by its column of the table."""
    slots = t.block_table[r, :-(-n // 16)].long().repeat_interleave(16)[:n] * 16 + torch.arange(n, device="cuda") % 16
    return [x.clone() for x in kv.read(slots)]


def test_park_and_resume():
    from paper_2512_04013_amd import runtime as rt
    kv, t = _kv(), rt.StepTables(3, 64, 20, POOL)
    t.update(i32([100, 77, 5]), i32([0, 0, 0]))
    before = [_rows(t, kv, r, n) for r, n in enumerate((100, 77, 5))]
    held = int(t.held[1])
    ids = t.block_table[1, :held].cpu().numpy()                  # read back: one copy and a wait
    host = kv.host_buffer(held)
    kv.park(ids, i32(ids), host)
    t.update(i32([100, 0, 5]), i32([0, 0, 0]))                   # its blocks are free
    assert t.held.tolist() == [7, 0, 1] and int(t.free_count) == POOL - 8
    t.update(i32([260, 0, 5]), i32([1, 0, 1]))                   # and are taken by others
    for p in (kv.k_cache, kv.v_cache):
        p[t.block_table[0, 7:17].long()] = 0.0
    t.update(i32([100, 77, 5]), i32([0, 0, 0]))
    again = t.block_table[1, :held].cpu().numpy()
    kv.resume(again, i32(again), host)
    torch.cuda.synchronize()
    for r, n in enumerate((100, 77, 5)):
        assert all(torch.equal(a, b) for a, b in zip(_rows(t, kv, r, n), before[r])), r


def test_prompts_planned_on_the_host_then_drafts():
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(3)
    lengths = [130, 1, 95]
    rows = sum(lengths)
    q, k, v = (torch.randn(rows, h, D, generator=gen, device="cuda").to(torch.bfloat16) for h in (8, HKV, HKV))
    q_start = np.concatenate([[0], np.cumsum(lengths)])
    outs = []
    free = torch.randperm(POOL, generator=gen, device="cuda").to(torch.int32)
    for order in (torch.arange(POOL, dtype=torch.int32, device="cuda"), free):
        kv, t = _kv(1), rt.StepTables(3, rows, 20, POOL, max_draft=0, free_ids=order.clone())
        t.update(i32([0, 0, 0]), i32(lengths))
        kv.append_rows(t.slots, k, v)
        held = t.held.tolist()
        ids = torch.cat([t.block_table[r, :n] for r, n in enumerate(held)])
        att = rt.MixedAttention(kv.shape, kv, q_start, lengths, np.concatenate([[0], np.cumsum(held)]), ids.cpu().numpy(), ids)
        outs.append(att.run(q).clone())
    assert torch.equal(*outs)
    # tables with masks take over, with the free blocks as they are; a row a request is what the host's plan gives
    t2 = rt.StepTables(3, 12, 20, POOL, max_draft=4, block_table=t.block_table, held=t.held, free_ids=t.free_ids,
                       free_count=int(t.free_count))
    t2.update(t.kv_len, i32([1, 1, 1]))
    assert t2.state.tolist() == [0, 0, 0] and t2.kv_len.tolist() == [n + 1 for n in lengths]
    kv.append_rows(t2.slots, torch.zeros(12, HKV, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(12, HKV, D, dtype=torch.bfloat16, device="cuda"),
                   live_rows=t2.live_rows)
    tree = rt.TreeAttention(kv.shape, kv, t2)
    tree.plan()
    qs = torch.zeros(12, 8, D, dtype=torch.bfloat16, device="cuda")
    qs[:3] = q[:3]
    got = tree.run(qs)[:3].float()
    held = t2.held.tolist()
    ids = torch.cat([t2.block_table[r, :n] for r, n in enumerate(held)])
    att = rt.MixedAttention(kv.shape, kv, [0, 1, 2, 3], [n + 1 for n in lengths], np.concatenate([[0], np.cumsum(held)]), ids.cpu().numpy(), ids)
    want = att.run(q[:3].contiguous()).float()
    # both within 2^-8 of the sum of |p v| (bf16 probabilities), 2^-8 of the result and little else: values are a few
    assert (got - want).abs().max() <= 2 * 2.0 ** -7 * float(v.float().abs().max())
