"""Rotary positions on the GPU: rows against float64, their gradient, and rows
rotated into the slots of every cache format."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402
from oracle import rope as orope  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

SCALINGS = {
    "plain": dict(),
    "linear": dict(scaling="linear", factor=4.0),
    "bands": dict(base=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original_len=8192),
    "ramp": dict(base=1e6, scaling="ramp", factor=4.0, low=1.0, high=32.0, original_len=32768),
}


def _shape(kv="bf16", hq=8, hkv=2, d=128):
    io = "f32" if kv == "f32" else "bf16"
    return aug.make_shape(hq, hkv, d, io, kv, io, 0.1)


def _rope(dim, interleaved=False, magnitude=1.0, **kw):
    from paper_2512_04013_amd import runtime as rt
    return rt.Rope(dim, interleaved=interleaved, magnitude=magnitude, **kw), orope.frequencies(dim, **kw)


def _rows(gen, n, heads, d, dtype, pad=0):
    """Rows `pad` elements further apart than they are long; NaN between them."""
    t = torch.full((n, heads * d + pad), float("nan"), device="cuda", dtype=dtype)
    t[:, :heads * d] = torch.randn(n, heads * d, generator=gen, device="cuda").to(dtype)
    return t[:, :heads * d].view(n, heads, d)


def _error(x, positions, w, interleaved, magnitude):
    """Result in float64 and how far a float32 rotation may be off.

    Cosine and sine: the angle, at most pi/4 < 1, is rounded once (2^-25), the series cut
    off (2e-9 < 2^-28) and its value rounded a few times around magnitudes of at most 1 (below 2^-24
    together): off by less than 2^-23, and with the magnitude's product rounded by
    2^-23 + 2^-24. A product and a sum on top: 2^-24 of the product, 2^-24 of the result. With
    x and x' the pair, m the magnitude: m (|x| + |x'|) (2^-23 + 2^-24 + 2^-24) + 2^-24 |y|. The
    oracle's own angle, a product in float64 of up to 2^31 positions and w <= 1, is off by up to
    2^31 * 2^-53 = 2^-22, and so is the library's in turns: only where positions are that far."""
    y = orope.rotate(x, positions, w, interleaved, magnitude)
    half = len(w)
    both = np.zeros_like(x)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    both[..., a] = both[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far = (np.abs(positions.astype(np.float64))[:, None] * np.abs(w) * 2.0 ** -52 * 2 * np.pi)
    angle = np.zeros((len(positions), 1, x.shape[-1]))
    angle[:, 0, a] = angle[:, 0, b] = far
    return y, abs(magnitude) * both * (2.0 ** -22 + angle) + 2.0 ** -24 * np.abs(y)


def _close(got, y, bound, dtype, what):
    got = got.double().cpu().numpy()
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(y) + bound)
    worst = float((np.abs(got - y) / np.maximum(bound, 1e-300)).max()) if got.size else 0.0
    say(f"  {what}: {worst:.3f} of the bound")
    assert (np.abs(got - y) <= bound).all(), (what, worst)


@pytest.mark.parametrize("kv,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("name", SCALINGS)
def test_rows(kv, d, interleaved, name):
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = torch.float32 if kv == "f32" else torch.bfloat16
    for dim, n, hq, hkv, pad, mag in ((d, 37, 8, 2, 0, 1.0), (16, 1, 1, 1, 8, 1.25), (48, 5, 3, 3, 40, -0.5), (d // 2, 300, 16, 4, 64, 1.0)):
        rope, w = _rope(dim, interleaved, mag, **SCALINGS[name])
        pos = torch.randint(-1000, 1 << 20, (n,), generator=gen, device="cuda", dtype=torch.int32)
        pos[0] = 0
        q, k = _rows(gen, n, hq, d, dtype, pad), _rows(gen, n, hkv, d, dtype, pad)
        shape = _shape(kv, hq, hkv, d)
        qo, ko = rt.rope_rows(shape, rope, pos, q, k)
        for x, got in ((q, qo), (k, ko)):
            y, bound = _error(x.double().cpu().numpy(), pos.cpu().numpy(), w, interleaved, mag)
            _close(got, y, bound, dtype, f"{kv} d{d} {name} dim {dim} rows {n}")
        # one alone, into strided rows, in place: the same bits, and nothing between the rows
        ko2 = _rows(gen, n, hkv, d, dtype, pad)
        assert rt.rope_rows(shape, rope, pos, None, k, k_out=ko2)[0] is None
        assert torch.equal(ko2, ko)
        base = q.as_strided((n, q.stride(0)), (q.stride(0), 1)) if pad and n > 1 else None
        rt.rope_rows(shape, rope, pos, q, q_out=q)
        assert torch.equal(q, qo)
        if base is not None:
            assert base[:-1, hq * d:].isnan().all()


def test_far_positions():
    """The largest positions, whose angles are off by what the product in float64 leaves."""
    from paper_2512_04013_amd import runtime as rt
    rope, w = _rope(128)
    gen = torch.Generator(device="cuda").manual_seed(2)
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 24, 2 ** 24 - 1, -1, 0, 1], dtype=torch.int32, device="cuda")
    x = _rows(gen, len(pos), 2, 128, torch.float32)
    got = rt.rope_rows(_shape("f32"), rope, pos, k=x)[1]
    _close(got, *_error(x.double().cpu().numpy(), pos.cpu().numpy(), w, False, 1.0), torch.float32, "far")


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """Negated positions against the formula's gradient and against differences."""
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(3)
    rope, w = _rope(32, interleaved, 1.5)
    n, heads, d = 9, 2, 64
    shape = _shape("f32", heads, heads, d)
    pos = torch.randint(0, 5000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    x, g = _rows(gen, n, heads, d, torch.float32), _rows(gen, n, heads, d, torch.float32)
    back = rt.rope_rows(shape, rope, -pos, g)[0]
    # the formula: dx = m (g cos + g' sin, g' cos - g sin)
    a = pos.double()[:, None, None] * torch.from_numpy(w).cuda()
    c, s = 1.5 * torch.cos(a), 1.5 * torch.sin(a)
    gd = g.double()
    lo, hi = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    want = gd.clone()
    want[..., lo], want[..., hi] = gd[..., lo] * c + gd[..., hi] * s, gd[..., hi] * c - gd[..., lo] * s
    _, bound = _error(g.double().cpu().numpy(), -pos.cpu().numpy(), w, interleaved, 1.5)
    _close(back, want.cpu().numpy(), bound, torch.float32, "gradient")
    # differences of sum(g * rotate(x)), which is linear in x: a step of 1 in one dim changes it by the gradient's element.
    # Both sums have 2 n d elements of size ~1 rounded in float64; the rotation's own rounding is what counts:
    # two of the bounds of a pair of elements, each times |g|.
    base = rt.rope_rows(shape, rope, pos, x)[0].double()
    for r, h, e in ((0, 0, 0), (3, 1, 17), (8, 0, 31), (5, 1, 40)):
        moved = x.clone()
        moved[r, h, e] += 1.0
        step = float(moved[r, h, e].double() - x[r, h, e].double())
        change = float(((rt.rope_rows(shape, rope, pos, moved)[0].double() - base) * gd).sum()) / step
        tol = 4 * 1.5 * 2.0 ** -22 * (float(x[r, h].abs().max()) + 2.0) * float(g[r, h].abs().max()) * 2 / step
        assert abs(change - float(back[r, h, e])) <= tol, (r, h, e, change, float(back[r, h, e]), tol)


# ---- into the cache ------------------------------------------------------------------------

FORMATS = [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128), ("fp8", 128), ("fp4", 128)]


def _pool(kv, blocks, hkv, d, gen):
    """A pool whose every slot holds something (a NaN bit pattern would do as well, but must not move)."""
    if kv == "fp4":
        pools = [torch.randint(0, 256, (blocks, hkv * 1088), generator=gen, device="cuda").to(torch.uint8) for _ in range(2)]
        return pools, [None, None]
    if kv == "fp8":
        pools = [torch.randint(0, 126, (blocks, hkv, 16, d), generator=gen, device="cuda").to(torch.uint8) for _ in range(2)]
        return pools, [torch.rand(blocks, hkv, generator=gen, device="cuda") * 0.01 for _ in range(2)]
    dtype = torch.float32 if kv == "f32" else torch.bfloat16
    return [torch.randn(blocks, hkv, 16, d, generator=gen, device="cuda").to(dtype) for _ in range(2)], [None, None]


def _kv(shape, pools, scales):
    from paper_2512_04013_amd import runtime as rt
    return rt.PagedKV(shape, *pools, *scales, staging_bytes=1)


def _copy(x):
    return [None if t is None else t.clone() for t in x]


@pytest.mark.parametrize("kv,d", FORMATS)
def test_append_by_slots_is_the_planned_append(kv, d):
    """Without a rope, bit for bit what the append of a planned batch writes, whole pools compared."""
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(4)
    for q_len, ctx, hkv in (([1, 5, 40, 16], [1, 21, 100, 32], 3), ([1], [17], 1), ([1] * 9, list(range(1, 10)), 8), ([130], [131], 2)):
        shape = _shape(kv, hkv * 2, hkv, d)
        nblk = [-(-c // 16) for c in ctx]
        blocks = sum(nblk) + 5
        perm = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
        ids = perm[:sum(nblk)].contiguous()
        pools, scales = _pool(kv, blocks, hkv, d, gen)
        mine = _kv(shape, _copy(pools), _copy(scales))
        planned = _kv(shape, _copy(pools), _copy(scales))
        q_start, bt = np.concatenate([[0], np.cumsum(q_len)]), np.concatenate([[0], np.cumsum(nblk)])
        dtype = torch.float32 if kv == "f32" else torch.bfloat16
        k, v = (_rows(gen, sum(q_len), hkv, d, dtype, 8 * i) * 3 for i in range(2))
        att = rt.MixedAttention(shape, planned, q_start, ctx, bt, ids.cpu().numpy(), ids)
        att.append(k.contiguous(), v.contiguous())
        host = ids.cpu().numpy()
        slots = [int(host[bt[r] + p // 16]) * 16 + p % 16 for r in range(len(ctx)) for p in range(ctx[r] - q_len[r], ctx[r])]
        assert mine.append_rows(torch.tensor(slots, device="cuda"), k, v) is None
        for a, b in ((mine.k_cache, planned.k_cache), (mine.v_cache, planned.v_cache)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (kv, d, hkv)
        if kv == "fp8":
            assert torch.equal(mine.k_scale, planned.k_scale) and torch.equal(mine.v_scale, planned.v_scale)


@pytest.mark.parametrize("kv,d", FORMATS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_append(kv, d, interleaved):
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(5)
    for n, hq, hkv, dim in ((1, 2, 1, 64), (33, 16, 2, 16), (97, 32, 8, d)):
        rope, w = _rope(dim, interleaved, 1.125, **SCALINGS["bands"])
        shape = _shape(kv, hq, hkv, d)
        blocks = n + 7
        pools, scales = _pool(kv, blocks, hkv, d, gen)
        pool = _kv(shape, _copy(pools), _copy(scales))
        # runs of a block each: whole, from the middle, and single slots; two rows go nowhere
        perm = torch.randperm(blocks, generator=gen, device="cuda").tolist()
        slots, at = [], 0
        while len(slots) < n:
            first = int(torch.randint(0, 16, (1,), generator=gen, device="cuda"))
            first = 0 if at % 3 == 0 else first
            slots += [perm[at] * 16 + t for t in range(first, min(16, first + n - len(slots)))]
            at += 1
        if n > 30:
            slots[3], slots[20] = -1, blocks * 16
        live = [i for i, s in enumerate(slots) if 0 <= s < blocks * 16]
        slots = torch.tensor(slots, device="cuda")
        pos = torch.randint(0, 200000, (n,), generator=gen, device="cuda", dtype=torch.int32)
        dtype = torch.float32 if kv == "f32" else torch.bfloat16
        qkv = _rows(gen, n, hq + 2 * hkv, d, dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q_out = pool.append_rows(slots, k, v, q=q, rope=rope, positions=pos)
        wq, wk = rt.rope_rows(shape, rope, pos, q, k)
        assert torch.equal(q_out, wq)
        got_k, got_v = pool.read(slots)
        y, bound = _error(k.double().cpu().numpy(), pos.cpu().numpy(), w, interleaved, 1.125)
        for name, got, want, off, raw in (("k", got_k, y, bound, wk), ("v", got_v, v.double().cpu().numpy(), 0.0, v)):
            assert (got[[i for i in range(n) if i not in live]] == 0).all()
            if kv in ("f32", "bf16"):
                assert torch.equal(got[live], raw[live])
                continue
            g = got.double().cpu().numpy()[live]
            want = want[live]
            off = np.broadcast_to(off, y.shape)[live]
            if kv == "fp4":
                # half the distance of levels around, in units of the group's power of two; saturation takes at most 1
                a = np.abs(want.reshape(len(live), hkv, 4, 32)).max(-1, keepdims=True)
                e = np.floor(np.log2(np.maximum(a, 1e-30)))
                unit = 2.0 ** (np.where(a >= 1.75 * 2.0 ** e * (1 - 2.0 ** -20), e + 1, e) - 2)
                m = np.abs(want.reshape(unit.shape[:-1] + (32,))) / unit
                half = np.where(m <= 2, 0.25, np.where(m <= 4, 0.5, 1.0)) * unit * (1 + 2.0 ** -18)
                half = half.reshape(want.shape)
            else:
                # half a step of E4M3 (2^-4 of the value, 2^-10 of the scale below 2^-6), the reading's bf16
                s = (pool.k_scale if name == "k" else pool.v_scale).double().cpu().numpy()
                s = s[slots.cpu().numpy()[live] // 16][:, :, None]
                half = np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
            worst = (np.abs(g - want) / (half + 2 * off + 1e-30)).max()
            say(f"  {kv} {name} rows {n}: {worst:.3f} of the bound")
            assert worst <= 1.0
        # what no slot names is as it was
        untouched = sorted(set(range(blocks)) - {int(s) // 16 for s in slots.tolist() if s >= 0})
        for a, b in ((pool.k_cache, pools[0]), (pool.v_cache, pools[1])):
            assert torch.equal(a[untouched].view(torch.uint8), b[untouched].view(torch.uint8))


@pytest.mark.parametrize("kv,d", FORMATS)
def test_rows_move_within_a_cache(kv, d):
    """Drafts that were accepted move down to the slots behind the context: read, then append by slots."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    hkv = 2
    pools, scales = _pool(kv, 6, hkv, d, gen)
    if kv == "fp4":
        for p in pools:                                    # scales that the append writes
            p[:, hkv * 1024:] = 120
    pool = _kv(_shape(kv, 4, hkv, d), pools, scales)
    src = torch.tensor([16 * 3 + 13, 16 * 3 + 15, 16 * 1 + 2, 16 * 1 + 9], device="cuda")
    dst = torch.tensor([16 * 3 + 12, 16 * 3 + 13, 16 * 3 + 14, 16 * 3 + 15], device="cuda")
    rows = pool.read(src)
    before = [t.clone() for t in rows]
    pool.append_rows(dst, *rows)
    for got, want in zip(pool.read(dst), before):
        if kv == "fp8":
            # encoded anew under the block's scale: half a step of it, and bf16 once more
            assert ((got - want).abs().float() <= want.abs().float() * (2.0 ** -4 + 2.0 ** -7) + 0.02 * 2.0 ** -9).all()
        elif kv == "fp4":
            # a group may hold less than its scale allows: a finer scale, the same or nearer values
            assert ((got - want).abs() <= 0).all()
        else:
            assert torch.equal(got, want)


def test_replays_and_streams():
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(7)
    rope, _ = _rope(128)
    shape = _shape("fp8", 16, 2)
    pools, scales = _pool("fp8", 40, 2, 128, gen)
    a, b = _kv(shape, _copy(pools), _copy(scales)), _kv(shape, _copy(pools), _copy(scales))
    n = 24
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    q, k, v = (_rows(gen, n, h, 128, torch.bfloat16) for h in (16, 2, 2))
    q_out = torch.empty_like(q)
    slots.fill_(-1)
    a.append_rows(slots, k, v, q=q, rope=rope, positions=pos, q_out=q_out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.append_rows(slots, k, v, q=q, rope=rope, positions=pos, q_out=q_out)
    side = torch.cuda.Stream()
    for step in range(3):
        first = int(torch.randint(0, 40 * 16 - n, (1,), generator=gen, device="cuda"))
        slots.copy_(torch.arange(first, first + n, device="cuda"))
        pos.copy_(torch.randint(0, 9999, (n,), generator=gen, device="cuda", dtype=torch.int32))
        k.normal_(generator=gen)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = b.append_rows(slots, k, v, q=q, rope=rope, positions=pos)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want)
        assert torch.equal(a.k_cache, b.k_cache) and torch.equal(a.k_scale, b.k_scale)
        assert torch.equal(a.v_cache, b.v_cache) and torch.equal(a.v_scale, b.v_scale)


def test_rows_of_an_fp8_block_in_any_order():
    """Order within a block, rows that go nowhere between them, however many, and what call they share change no bit."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    hkv = 3
    pools, scales = _pool("fp8", 5, hkv, 128, gen)
    shape = _shape("fp8", 3, hkv)
    plain, mixed = _kv(shape, _copy(pools), _copy(scales)), _kv(shape, _copy(pools), _copy(scales))
    groups = [[33, 34, 37, 47], [48], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15], [70, 79], [16, 20]]
    k, v = (_rows(gen, sum(map(len, groups)), hkv, 128, torch.bfloat16) * 5 for _ in range(2))
    at, slots, order = 0, [], []
    for g in groups:
        rows = list(range(at, at + len(g)))
        plain.append_rows(torch.tensor(g, device="cuda"), k[rows], v[rows])
        at += len(g)
        perm = torch.randperm(len(g), generator=gen, device="cuda").tolist()
        for i in perm:
            gap = [0, 1, 70, 200][len(slots) % 4]
            slots += [-1, 80, 1 << 40, -5][:1] * gap + [g[i]]
            order += [0] * gap + [rows[i]]
    mixed.append_rows(torch.tensor(slots, device="cuda"), k[order], v[order])
    for a, b in ((plain.k_cache, mixed.k_cache), (plain.v_cache, mixed.v_cache), (plain.k_scale, mixed.k_scale), (plain.v_scale, mixed.v_scale)):
        assert torch.equal(a, b)
    assert not torch.equal(plain.k_cache, pools[0])


@pytest.mark.parametrize("kv,d", FORMATS)
def test_live_rows(kv, d):
    """Rows from live_rows on are as if they were not there, in every tensor: their slots are others' slots."""
    from paper_2512_04013_amd import runtime as rt
    gen = torch.Generator(device="cuda").manual_seed(9)
    hkv, dtype, rope = 2, torch.float32 if kv == "f32" else torch.bfloat16, rt.Rope(d)
    shape = _shape(kv, 4, hkv, d)
    pools, scales = _pool(kv, 40, hkv, d, gen)
    for n in (3, 40, 600):
        slots = torch.arange(n, device="cuda") + 5
        pos = torch.arange(n, dtype=torch.int32, device="cuda")
        k, v, q = (_rows(gen, n, h, d, dtype) for h in (hkv, hkv, 4))
        for live in (-1, 0, 1, n // 2, n - 1, n, n + 1):
            m = min(max(live, 0), n)
            a, b = (_kv(shape, _copy(pools), _copy(scales)) for _ in range(2))
            stale = slots.clone()
            stale[m:] = slots[:n - m] if m else slots       # of live rows
            out = torch.full((n, 4, d), 3.0, dtype=dtype, device="cuda")
            a.append_rows(stale, k, v, q=q, rope=rope, positions=pos, q_out=out, live_rows=torch.tensor([live], dtype=torch.int32, device="cuda"))
            want = torch.full_like(out, 3.0)
            if m:
                want[:m] = b.append_rows(slots[:m], k[:m], v[:m], q=q[:m], rope=rope, positions=pos[:m])
            assert torch.equal(out, want), (n, live)
            for x, y in ((a.k_cache, b.k_cache), (a.v_cache, b.v_cache), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
                assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (n, live)


@pytest.mark.parametrize("rows,hkv", [(1100, 8), (2500, 8), (9000, 8), (40000, 1)])
def test_many_rows_into_an_fp8_cache(rows, hkv):
    """Waves that look for blocks among several rows: blocks that begin or go on in another wave's rows, rows that go
    nowhere, rows behind the last; bit for bit what one call a request writes."""
    rng = random.Random(rows)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    blocks = rows // 8 + 300
    pools, scales = _pool("fp8", blocks, hkv, 128, gen)
    shape = _shape("fp8", hkv, hkv)
    one, each = _kv(shape, _copy(pools), _copy(scales)), _kv(shape, _copy(pools), _copy(scales))
    free = list(range(blocks))
    rng.shuffle(free)
    slots, ends = [], []
    while len(slots) < rows - 300 and len(free) > 20:
        n, first = rng.choice([1, 1, 3, 16, 30, 100, 270]), rng.randrange(16)
        ids = [free.pop() for _ in range(-(-(first + n) // 16))]
        slots += [ids[(first + i) // 16] * 16 + (first + i) % 16 for i in range(n)]
        slots += [-1] * rng.choice([0, 0, 1, 20, 130])
        ends.append(len(slots))
    live = len(slots)
    slots += slots[:rows - live]
    k, v = (_rows(gen, rows, hkv, 128, torch.bfloat16) for _ in range(2))
    slots = torch.tensor(slots, device="cuda")
    one.append_rows(slots, k, v, live_rows=torch.tensor([live], dtype=torch.int32, device="cuda"))
    for a, b in zip([0] + ends, ends):
        each.append_rows(slots[a:b].contiguous(), k[a:b], v[a:b])
    for a, b in ((one.k_cache, each.k_cache), (one.v_cache, each.v_cache), (one.k_scale, each.k_scale), (one.v_scale, each.v_scale)):
        assert torch.equal(a, b)
    assert not torch.equal(one.k_cache, pools[0])
