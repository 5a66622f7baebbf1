"""Attention of drafts into its own queries: the bits of a run into another tensor, for requests in one span and in
several, and for every number of waves that share a request's columns."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_tree import LAYERS, Case  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

PICK = [0, 1, 3, 5, 9, 12]


@pytest.mark.parametrize("layer", [LAYERS[i] for i in PICK], ids=["-".join(map(str, LAYERS[i])) for i in PICK])
def test_in_place(layer):
    for rows, ctx in (([5, 1, 40, 64], [60, 1, 90, 64]), ([64, 33, 2], [4100, 9000, 20000])):
        c = Case(layer, rows, ctx, seed=3)
        n = sum(rows)
        c.att.plan()
        want = c.att.run(c.q)[:n].clone()
        for _ in range(3):
            q = c.q.clone()
            assert c.att.run(q, out=q) is q
            assert torch.equal(q[:n], want) and q[n:].isnan().all()


def test_part_of_the_queries_is_refused():
    import paper_2512_04013_amd as aug
    c = Case(LAYERS[5], [5, 3], [60, 9], seed=3)
    c.att.plan()
    rows = c.q.shape[0]
    both = torch.zeros(rows + 2, *c.q.shape[1:], dtype=c.q.dtype, device="cuda")
    with pytest.raises(aug.AugError):
        c.att.run(both[:rows], out=both[2:])
    assert not both.any()
