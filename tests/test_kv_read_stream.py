"""Rows that a read allocates itself come from the stream that writes them."""

import contextlib
import os

import pytest

import paper_2512_04013_amd as aug

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")


def _pool(rt, device="cpu"):
    s = aug.make_shape(6, 3, 128, "bf16", "fp4", "bf16", 0.1)
    pool = torch.full((4, 3 * 1088), 127, dtype=torch.uint8, device=device)
    return rt.PagedKV(s, pool, pool.clone(), staging_bytes=1)


def test_allocations_are_made_under_the_given_stream(monkeypatch):
    """On the CPU: which stream is torch's current one at each allocation."""
    from paper_2512_04013_amd import runtime as rt
    kv = _pool(rt)
    current, made, calls = ["caller"], [], []

    @contextlib.contextmanager
    def under(stream):
        current.append(stream)
        yield
        current.pop()

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: ("handle", handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (made.append(current[-1]), empty(*a, **k))[1])
    monkeypatch.setattr(rt, "aug_kv_read", lambda *a, stream=None: calls.append((current[-1], stream)))
    slots = torch.zeros(5, dtype=torch.int64)

    def streams(**kw):
        made.clear()
        k, v = kv.read(slots, **kw)
        assert k.shape == v.shape == (5, 3, 128)
        return made

    assert streams() == ["caller"] * 2
    assert streams(stream="side") == ["side"] * 2
    assert streams(stream=77) == [("handle", 77)] * 2
    assert streams(stream=0) == ["default"] * 2
    rows = empty(5, 3, 128, dtype=torch.bfloat16)
    assert streams(k_out=rows, stream="side") == ["side"]
    assert streams(k_out=rows, v_out=rows.clone(), stream="side") == []
    assert current == ["caller"] and [c[1] for c in calls] == [None, "side", 77, 0, "side", "side"]


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("raw", [False, True])
def test_rows_read_on_a_side_stream(raw):
    """Memory that the current stream has just given back, with work still queued
    on it, is not what a side stream writes."""
    from paper_2512_04013_amd import runtime as rt
    kv = _pool(rt, "cuda")
    kv.k_cache[:, :3 * 1024] = 0x12
    kv.v_cache[:, :3 * 1024] = 0x21
    slots = torch.arange(64, device="cuda").repeat(500)
    want_k, want_v = kv.read(slots)
    want_k, want_v = want_k.clone(), want_v.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        for _ in range(4):
            busy = busy @ busy * 1e-3
        old = [torch.empty_like(want_k) for _ in range(4)]
        for t in old:
            t.fill_(7.0)                        # queued behind the products
        del old, t
        k, v = kv.read(slots, stream=side.cuda_stream if raw else side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(k, want_k) and torch.equal(v, want_v)
        del k, v
    assert want_k.abs().sum() > 0
