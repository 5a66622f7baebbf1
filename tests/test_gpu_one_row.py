"""One token's rows as a program has them: transposed from [heads][1][dim], expanded, or with a stride
that means nothing; the same bits as from a contiguous row, out of place, in place and into the cache."""

import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

VIEWS = [lambda x: x[0].clone().unsqueeze(1).transpose(0, 1), lambda x: x.clone().as_strided(x.shape, (7, x.shape[2], 1)),
         lambda x: x[0].clone().unsqueeze(0), lambda x: x.clone().expand(1, -1, -1)]


@pytest.mark.parametrize("kv,d", [("f32", 64), ("bf16", 128), ("fp8", 128), ("fp4", 128)])
@pytest.mark.parametrize("view", range(len(VIEWS)))
def test_one_row(kv, d, view):
    from paper_2512_04013_amd import runtime as rt
    io = "f32" if kv == "f32" else "bf16"
    dtype = torch.float32 if kv == "f32" else torch.bfloat16
    shape, rope, like = aug.make_shape(8, 2, d, io, kv, io, 0.1), rt.Rope(d), VIEWS[view]
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1, h, d, generator=gen, device="cuda").to(dtype) for h in (8, 2, 2))
    pos, slot = torch.tensor([77], dtype=torch.int32, device="cuda"), torch.tensor([2 * 16 + 5], device="cuda")
    want = rt.rope_rows(shape, rope, pos, q, k)
    got = rt.rope_rows(shape, rope, pos, like(q), like(k))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    inplace = like(q)
    assert torch.equal(rt.rope_rows(shape, rope, pos, inplace, q_out=inplace)[0], want[0])

    def pool():
        if kv == "fp4":
            return [torch.zeros(4, 2 * aug.MXFP4_CELL_BYTES, dtype=torch.uint8, device="cuda") for _ in range(2)]
        if kv == "fp8":
            return [torch.zeros(4, 2, 16, d, dtype=torch.uint8, device="cuda") for _ in range(2)] + \
                   [torch.zeros(4, 2, device="cuda") for _ in range(2)]
        return [torch.zeros(4, 2, 16, d, dtype=dtype, device="cuda") for _ in range(2)]

    a, b = pool(), pool()
    out = rt.PagedKV(shape, *a, staging_bytes=1).append_rows(slot, k, v, q=q, rope=rope, positions=pos)
    other = rt.PagedKV(shape, *b, staging_bytes=1).append_rows(slot, like(k), like(v), q=like(q), rope=rope, positions=pos)
    assert torch.equal(out, other) and torch.equal(out, want[0])
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and a[0].any()
