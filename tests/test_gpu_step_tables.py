"""A step's tables on the GPU against lists and loops, exactly: many steps on end,
requests that are refused, odd lengths, and replays of a captured step."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402
from oracle import steps  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731


class Pair:
    """The device's tables and the plain ones, from the same start."""

    def __init__(self, reqs, rows, width, pool, max_draft, seed=0):
        from paper_2512_04013_amd import runtime as rt
        rng = random.Random(seed)
        free = list(range(pool))
        rng.shuffle(free)
        self.t = rt.StepTables(reqs, rows, width, pool, max_draft=max_draft, free_ids=i32(free))
        self.s = steps.State([[] for _ in range(reqs)], free)

    def step(self, ctx, q, parents=None, stream=None):
        t = self.t
        for x in (t.positions, t.slots, t.seen):
            if x is not None:
                x.fill_(-7)
        self.want = steps.update(self.s, ctx, q, parents, t.max_rows, t.max_blocks, t.max_draft)
        t.update(i32(ctx), i32(q), None if parents is None else i32(parents), stream=stream)
        self.check()
        return self.want

    def check(self):
        t, want = self.t, self.want
        for name in ("q_start", "kv_len", "state"):
            assert getattr(t, name).tolist() == want[name], name
        rows = want["q_start"][-1]
        for name in ("positions", "slots") + (("seen",) if t.max_draft else ()):
            got = getattr(t, name).tolist()
            assert got[:rows] == [v - (1 << 64) if v >> 63 == 1 else v for v in want[name]], name
            assert set(got[rows:]) <= {-7}, name + " behind the last row"
        assert t.held.tolist() == [len(x) for x in self.s.table]
        table = t.block_table.cpu().numpy()
        for r, ids in enumerate(self.s.table):
            assert table[r, :len(ids)].tolist() == ids, r
        n = int(t.free_count)
        assert t.free_ids[:n].tolist() == self.s.free
        assert int(t._scratch.sum()) == 0


def tree(rng, q, invalid=False):
    out = []
    for n in q:
        out += [rng.choice([-1, i, i + 1, 99, -5]) if invalid and rng.random() < 0.2 else rng.randint(-1, i - 1) if i else -1
                for i in range(max(n, 0))]
    return out


@pytest.mark.parametrize("reqs,draft,width,pool,steps_", [(1, 64, 9, 9, 12), (2, 1, 3, 8, 12), (7, 8, 20, 64, 25), (63, 5, 12, 500, 10),
                                                           (257, 33, 40, 6000, 8), (1025, 3, 10, 4000, 5), (4096, 2, 4, 9000, 3)])
@pytest.mark.parametrize("seed", [0, 1])
def test_many_steps(reqs, draft, width, pool, steps_, seed):
    rng = random.Random(seed)
    say(f"[tables] {reqs} requests of up to {draft} rows, {width} columns, seed {seed}")
    rows = reqs * draft
    p = Pair(reqs, rows, width, pool, draft, seed)
    ctx = [0] * reqs
    for _ in range(steps_):
        q = [rng.choice([0, 1, draft, rng.randint(0, draft)]) for _ in range(reqs)]
        parents = tree(rng, q, invalid=seed == 1) if rng.random() < 0.7 else None
        if parents is not None:
            parents += [-1] * (rows - len(parents))
        want = p.step(ctx, q, parents)
        for r in range(reqs):
            if rng.random() < 0.05:
                ctx[r] = 0                                     # ended
            elif want["state"][r] == steps.OK:
                ctx[r] = min(ctx[r] + rng.randint(0, q[r]), width * 16 - draft) + rng.choice([0, 0, 0, 17])
                ctx[r] = min(ctx[r], width * 16)


def test_invalid_requests():
    p = Pair(9, 20, 4, 12, 6)
    p.step([3, 10, 0, 0, 33, 5, 0, 0, 1], [2, 6, 0, 1, 1, 0, 0, 0, 0])
    # a negative context, a negative row count, too many rows, beyond the table, a context at the table's end
    p.step([-1, 10, 0, 60, 33, 64, 65, 7, 1], [2, -3, 7, 5, 1, 0, 0, 1, 0])
    assert p.want["state"] == [2, 2, 2, 2, 0, 0, 2, 0, 0]
    # rows beyond max_rows: the request that crosses is refused and so is every later one that has rows
    p.step([1] * 9, [6, 6, 6, 3, 0, 1, 0, 6, 0])
    assert p.want["state"] == [0, 0, 0, 2, 0, 2, 0, 2, 0] and p.want["q_start"][-1] == 20
    big = 2 ** 31 - 1
    p.step([big, 0, big, 0, 0, 0, -big - 1, 0, 0], [big, big, 0, 1, big, 0, -big - 1, big, big])
    assert p.want["state"] == [2, 2, 2, 2, 2, 0, 2, 2, 2]


def test_blocks_run_out():
    p = Pair(5, 10, 8, 6, 2)
    p.step([30, 30, 30, 0, 30], [2, 2, 2, 0, 2])
    assert p.want["state"] == [0, 0, 0, 0, 1]
    p.step([32, 0, 32, 0, 30], [1, 0, 1, 0, 2])              # two come back, two are taken, none is left for the last
    assert p.want["state"] == [0, 0, 0, 0, 1] and int(p.t.free_count) == 0
    p.step([32, 0, 0, 0, 30], [1, 0, 0, 0, 2])
    assert p.want["state"] == [0, 0, 0, 0, 0]


def test_held_out_of_range_is_refused():
    p = Pair(3, 6, 4, 12, 2)
    p.step([10, 20, 30], [1, 1, 1])
    p.t.held.copy_(i32([-1, 2, 5]))
    p.t.update(i32([10, 20, 30]), i32([2, 2, 2]))
    assert p.t.state.tolist() == [2, 0, 2] and p.t.held.tolist() == [-1, 2, 5]
    assert p.t.slots.tolist()[:2] == [-1, -1] and p.t.slots.tolist()[4:] == [-1, -1]


@pytest.mark.parametrize("reqs", [1, 5])
def test_long_prompts_without_masks(reqs):
    p = Pair(reqs, 6000, 500, 2600, 0)
    assert p.t.seen is None
    q = [4999, 0, 1, 700, 300][:reqs]
    p.step([17, 3, 0, 15, 16][:reqs], q)
    p.step([a + b for a, b in zip([17, 3, 0, 15, 16], q)], [1] * reqs)


def test_deepest_trees():
    """Chains of 64 rows, forwards, and trees whose paths are as long as they get."""
    p = Pair(3, 192, 8, 40, 64)
    p.step([5, 0, 63], [64, 64, 1])
    assert p.want["seen"][63] == 2 ** 64 - 1
    zigzag = [-1] + [max(i - 2, 0) for i in range(1, 64)]
    p.step([5, 0, 63], [64, 64, 64], list(range(-1, 63)) + zigzag + [-1] * 64)


def test_replays():
    """Two steps captured together, replayed with other lengths, eager work in between."""
    rng = random.Random(3)
    p = Pair(20, 160, 30, 500, 8)
    t = p.t
    ctx, q, ctx2, q2, parents = i32([0] * 20), i32([0] * 20), i32([0] * 20), i32([0] * 20), i32([-1] * 160)
    t.update(ctx, q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.update(ctx2, q2)
        t.update(ctx, q, parents)
    for _ in range(4):
        a, b = [rng.randint(0, 300) for _ in range(20)], [rng.randint(0, 400) for _ in range(20)]
        n = [rng.randint(0, 8) for _ in range(20)]
        tr = tree(rng, n)
        tr += [-1] * (160 - len(tr))
        for dst, src in ((ctx2, a), (ctx, b), (q, n), (parents, tr)):
            dst.copy_(i32(src))
        for x in (t.positions, t.slots, t.seen):
            x.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        steps.update(p.s, a, [0] * 20, None, 160, 30, 8)
        p.want = steps.update(p.s, b, n, tr, 160, 30, 8)
        p.check()


def test_another_stream():
    p = Pair(6, 24, 10, 50, 4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        p.step([3, 100, 0, 16, 15, 31], [4, 1, 4, 0, 2, 3])
    torch.cuda.synchronize()
    p.step([4, 101, 2, 16, 17, 32], [1] * 6, stream=torch.cuda.current_stream().cuda_stream)


def test_no_requests():
    from paper_2512_04013_amd import runtime as rt
    t = rt.StepTables(0, 4, 1, 1)
    t.update(i32([]), i32([]))
    assert t.q_start.tolist() == [0] and np.all(t.slots.cpu().numpy() == 0)
    with pytest.raises(aug.AugError):
        rt.StepTables(4097, 4, 1, 1).update(i32([0] * 4097), i32([0] * 4097))
