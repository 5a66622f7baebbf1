"""Plans of tree attention that are not of this call: of a batch of other sizes, of a step that was only
captured, and of memory that an earlier object's plan stood in. Nothing is read or written by them."""

import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402
from tests.test_gpu_tree import LAYERS, Case  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

PICK = [1, 5, 9, 12]       # fp32, bf16, fp8 and 4 bits, the last with 64 columns a wave


def _attend(c, plan, batch):
    att = c.att
    att.out.fill_(7.0)
    plan_bytes, workspace_bytes = aug.aug_tree_plan_size(c.shape, batch)
    big = torch.zeros(max(plan_bytes, plan.numel()), dtype=torch.uint8, device="cuda")
    big[:plan.numel()] = plan
    aug.aug_attn_tree(c.shape, batch, big, c.q.nan_to_num(), c.kv.k_cache, c.kv.v_cache, c.kv.k_scale, c.kv.v_scale,
                      c.kv.num_pool_blocks, att.out, torch.empty(workspace_bytes, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return att.out.clone()


@pytest.mark.parametrize("layer", [LAYERS[i] for i in PICK], ids=["-".join(map(str, LAYERS[i])) for i in PICK])
def test_batches_of_other_sizes(layer):
    c = Case(layer, [40, 3, 9], [700, 90, 300], seed=1)
    c.check("its own plan")
    plan, b = c.att.plan_dev, c.att._batch
    n = sum(c.rows)
    assert torch.equal(_attend(c, plan, b)[:n], c.att.run(c.q)[:n])
    for name, value in (("num_reqs", b.num_reqs - 1), ("max_rows", b.max_rows - 5), ("max_blocks", b.max_blocks - 1), ("max_draft", b.max_draft - 1),
                        ("max_draft", 1)):
        other = type(b)()
        C.memmove(C.byref(other), C.byref(b), C.sizeof(b))
        setattr(other, name, value)
        assert (_attend(c, plan, other) == 7.0).all(), name
    c.check("its own plan again")


def test_captured_plans_are_not_made_yet():
    """A run beside a plan that was only captured leaves the output alone, also in the memory of an earlier plan."""
    first = Case(LAYERS[5], [40, 3, 9], [700, 90, 300], seed=1)
    first.check("first")
    where = first.att.plan_dev.data_ptr()
    del first.att
    c = Case(LAYERS[5], [40, 3, 9], [400, 60, 200], seed=2)
    again = c.att.plan_dev.data_ptr() == where
    q = c.q.nan_to_num()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.att.plan()
        c.att.run(q)
    c.att.out.fill_(7.0)
    c.att.run(q)
    torch.cuda.synchronize()
    assert (c.att.out == 7.0).all(), again
    g.replay()
    torch.cuda.synchronize()
    n = sum(c.rows)
    replayed = c.att.out[:n].clone()
    assert (replayed != 7.0).any() and torch.equal(replayed, c.att.run(q)[:n])
