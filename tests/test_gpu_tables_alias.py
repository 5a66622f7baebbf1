"""Step tables whose context lengths are the lengths that the step before wrote, in place:
plain decoding and drafts, requests that are refused on the way, and replays, against lists and loops."""

import random

import pytest

torch = pytest.importorskip("torch")

from oracle import steps  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_step_tables import Pair, i32, tree  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _plain(p, q, parents):
    t = p.t
    p.want = steps.update(p.s, p.want["kv_len"], q, parents, t.max_rows, t.max_blocks, t.max_draft)


def _clear(t):
    for x in (t.positions, t.slots, t.seen):
        if x is not None:
            x.fill_(-7)


@pytest.mark.parametrize("reqs,draft,width,pool", [(1, 4, 9, 9), (64, 1, 12, 300), (64, 8, 12, 300), (300, 5, 20, 2500), (2000, 3, 10, 9000),
                                                   (4096, 2, 6, 9000)])
def test_lengths_in_place(reqs, draft, width, pool):
    rng = random.Random(reqs)
    say(f"[tables] {reqs} requests of up to {draft} rows, lengths in place")
    p = Pair(reqs, reqs * draft, width, pool, draft, seed=1)
    p.step([rng.randint(0, 16 * width - 8 * draft) for _ in range(reqs)], [draft] * reqs)
    refused = 0
    for k in range(8):
        q = [1 if draft == 1 else rng.randint(0, draft) for _ in range(reqs)]
        parents = tree(rng, q) if k % 2 else None
        if parents is not None:
            parents += [-1] * (reqs * draft - len(parents))
        _plain(p, q, parents)
        _clear(p.t)
        p.t.update(p.t.kv_len, i32(q), None if parents is None else i32(parents))
        p.check()
        refused += sum(s != steps.OK for s in p.want["state"])
    say(f"  {refused} refusals")
    assert refused or reqs in (1, 64)


def test_prompts_then_decodes():
    """Without masks: prompts of any length, then a row a request."""
    p = Pair(70, 9000, 40, 3000, 0, seed=2)
    rng = random.Random(2)
    p.step([0] * 70, [rng.randint(0, 120) for _ in range(70)])
    for _ in range(4):
        _plain(p, [1] * 70, None)
        _clear(p.t)
        p.t.update(p.t.kv_len, i32([1] * 70))
        p.check()


def test_replays_in_place():
    """Three decodes captured together, each after the one before, eager work between the replays."""
    p = Pair(200, 200, 30, 4000, 1, seed=3)
    p.step([7 * r % 300 for r in range(200)], [1] * 200)
    ones = i32([1] * 200)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            p.t.update(p.t.kv_len, ones)
    for _ in range(4):
        _clear(p.t)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for _ in range(3):
            _plain(p, [1] * 200, None)
        p.check()
        _plain(p, [1] * 200, None)
        p.t.update(p.t.kv_len, ones)
        p.check()


def test_other_overlaps_are_refused():
    import paper_2512_04013_amd as aug
    p = Pair(4, 16, 4, 16, 4)
    t, two = p.t, i32([1] * 4)
    for args in ((two, t.kv_len), (t.held, two), (t.state, two), (t.q_start[1:], two), (t.block_table[0], two), (two, two, t.positions),
                 (two, t.free_ids[:4])):
        with pytest.raises(aug.AugError):
            t.update(*args)
