"""Drafts over an fp8 cache, step after step: rows appended by slots, and those of an accepted path
read back and appended behind the context. After every call the whole pool, codes and scales, is
compared bit for bit with the formulas of aug.h, in float32 operations one by one; and every
committed row with what it was when it was committed.

Bound of the latter: a row is written twice (as a draft, and moved), and its block's codes are encoded anew whenever the
scale grows. Each encoding is off by half a step: 2^-4 of the value, or 2^-10 of the scale below its 2^-6; the
reading between them rounds to bf16 (2^-8). With s the largest scale that any block of the request has had, n
encodings leave at most n (2^-4 |x| 1.07^n + 2^-10 s) and 2^-8 |x|, where 1.07^n > (1 + 2^-4 + 2^-8)^n
stands for values that grew on the way."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2512_04013_amd as aug  # noqa: E402
from oracle.codecs import E4M3FN_TABLE, e4m3fn_encode  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

HKV, D = 2, 128
F32 = np.float32


class Plain:
    """A pool of K or V: codes and scales, and how often each block's codes have been rounded."""

    def __init__(self, codes, scale):
        self.codes, self.scale = codes.cpu().numpy().copy(), scale.cpu().numpy().copy()
        self.times = np.zeros(len(self.codes), int)
        self.largest = np.zeros_like(self.scale)

    def append(self, slots, x):
        """x [n, HKV, D] float32: the rows of a block together."""
        blocks = {}
        for i, s in enumerate(slots):
            if s >= 0:
                blocks.setdefault(s // 16, []).append((s % 16, i))
        for b, rows in blocks.items():
            at, rows = [s for s, _ in rows], [i for _, i in rows]
            self.times[b] = 1 if 0 in at else self.times[b] + 1
            for h in range(HKV):
                need, old = F32(np.abs(x[rows, h]).max()) / F32(448), self.scale[b, h]
                s = need if 0 in at else max(need, old)
                if 0 not in at and s > old:
                    others = [t for t in range(max(at)) if t not in at]
                    self.codes[b, h, others] = e4m3fn_encode(E4M3FN_TABLE[self.codes[b, h, others]].astype(F32) * old / s)
                self.codes[b, h, at] = e4m3fn_encode(x[rows, h] / s) if s > 0 else 0
                self.scale[b, h] = s
                self.largest[b, h] = max(s, self.largest[b, h])

    def read(self, slots):
        """float32 [n, HKV, D], as codes times scales, not rounded further."""
        b, t = np.array(slots) // 16, np.array(slots) % 16
        return E4M3FN_TABLE[self.codes[b, :, t]].astype(F32) * self.scale[b][:, :, None]


@pytest.mark.parametrize("seed", range(4))
def test_accepted_paths(seed):
    from paper_2512_04013_amd import runtime as rt
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    reqs, drafts, blocks = 5, 9, 60
    shape = aug.make_shape(2 * HKV, HKV, D, "bf16", "fp8", "bf16", 0.1)
    pools = [torch.randint(0, 126, (blocks, HKV, 16, D), generator=gen, device="cuda").to(torch.uint8) for _ in range(2)]
    scales = [torch.rand(blocks, HKV, generator=gen, device="cuda") * 0.01 for _ in range(2)]
    plain = [Plain(p, s) for p, s in zip(pools, scales)]
    kv = rt.PagedKV(shape, *pools, *scales, staging_bytes=1)
    ids = list(range(blocks))
    rng.shuffle(ids)
    table = [ids[12 * r:12 * r + 12] for r in range(reqs)]
    place = lambda r, j: table[r][j // 16] * 16 + j % 16  # noqa: E731
    dev = lambda a: torch.tensor(a, dtype=torch.int64, device="cuda")  # noqa: E731

    def same(what):
        torch.cuda.synchronize()
        for name, p, codes, scale in (("K", plain[0], kv.k_cache, kv.k_scale), ("V", plain[1], kv.v_cache, kv.v_scale)):
            assert np.array_equal(scale.cpu().numpy(), p.scale), (what, name)
            assert np.array_equal(codes.cpu().numpy(), p.codes), (what, name)

    ctx, first, moved, grown = [0] * reqs, [[[], []] for _ in range(reqs)], 0, 0
    for step in range(30):
        n = [rng.randint(0, drafts) if ctx[r] + drafts <= 192 else 0 for r in range(reqs)]
        slots = [place(r, ctx[r] + i) for r in range(reqs) for i in range(n[r])]
        if not slots:
            break
        size = 2.0 ** rng.randint(-3, 3)
        new = [(torch.randn(len(slots), HKV, D, generator=gen, device="cuda") * size).to(torch.bfloat16) for _ in range(2)]
        old = [p.scale.copy() for p in plain]
        kv.append_rows(dev(slots), *new)
        host = [x.float().cpu().numpy() for x in new]
        for p, x in zip(plain, host):
            p.append(slots, x)
        same(f"step {step}, drafts")
        grown += sum(int((p.scale > o).sum()) for p, o in zip(plain, old))
        # a path: the first row, and later ones in rising order
        source, target, at = [], [], 0
        for r in range(reqs):
            path = [0] + sorted(rng.sample(range(1, n[r]), rng.randint(0, n[r] - 1))) if n[r] else []
            source += [place(r, ctx[r] + i) for i in path] + [-1] * (n[r] - len(path))
            target += [place(r, ctx[r] + j) for j in range(len(path))] + [-1] * (n[r] - len(path))
            for k in range(2):
                first[r][k] += [host[k][at + i] for i in path]
            moved += sum(i != j for j, i in enumerate(path))
            ctx[r] += len(path)
            at += n[r]
        rows = kv.read(dev(source))
        live = [i for i, s in enumerate(source) if s >= 0]
        for p, x in zip(plain, rows):
            got, want = x.float().cpu().numpy()[live], torch.from_numpy(p.read([source[i] for i in live])).to(torch.bfloat16).float().numpy()
            assert np.array_equal(got, want), step
        kv.append_rows(dev(target), *rows)
        for p, x in zip(plain, rows):
            p.append(target, x.float().cpu().numpy())
        same(f"step {step}, moved")
    worst = 0.0
    for r in range(reqs):
        slots = [place(r, j) for j in range(ctx[r])]
        for k, p in enumerate(plain):
            if not slots:
                continue
            got, want = p.read(slots).astype(np.float64), np.stack(first[r][k]).astype(np.float64)
            block = np.array(slots) // 16
            n = (p.times[block] + 1)[:, None, None]           # and the drafts' own, before the block began anew
            s = p.largest[table[r]].max(0).astype(np.float64)[None, :, None]
            bound = n * (2.0 ** -4 * np.abs(want) * 1.07 ** n + 2.0 ** -10 * s) + 2.0 ** -8 * np.abs(want)
            worst = max(worst, float((np.abs(got - want) / bound).max()))
    say(f"[fp8 moves] seed {seed}: {moved} rows moved, {grown} scales grown, {worst:.3f} of the bound")
    assert moved > 20 and grown > 20 and worst <= 1.0
