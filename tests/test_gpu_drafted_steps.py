"""Steps of drafted tokens as a serving loop runs them, on the GPU from end to end: tables,
plan, append with rotary positions, tree attention, sampling, the longest accepted path,
and its rows moved behind the tokens before; captured once and replayed with other
drafts, requests that end, come anew and are refused for want of blocks.

After every replay each part is compared with its plain form, fed with what the parts before
it really put out. Bounds: attention as in attn_bound.py; a rotated value two products, their
sum and the angle (2^-22 of both its inputs), and one rounding to its type."""

import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import rope as orope  # noqa: E402
from oracle import sampling, steps  # noqa: E402
from oracle import tree as otree  # noqa: E402
from tests.attn_bound import within  # noqa: E402
from tests.gpu_util import say  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

REQS, DRAFTS, VOCAB, WIDTH, POOL = 5, 6, 11, 7, 9
ROWS = REQS * DRAFTS
LAYERS = {"f32": (8, 2, 64), "bf16": (8, 2, 128), "fp8": (8, 1, 128), "fp4": (4, 2, 128)}
BASE = 10000.0
f64 = lambda t: t.double().cpu().numpy()  # noqa: E731


class Loop:
    def __init__(self, kind):
        import paper_2512_04013_amd as aug
        from paper_2512_04013_amd import runtime as rt
        hq, hkv, d = LAYERS[kind]
        io = "f32" if kind == "f32" else "bf16"
        self.kind, self.hq, self.hkv, self.d = kind, hq, hkv, d
        self.dtype = torch.float32 if kind == "f32" else torch.bfloat16
        self.shape = aug.make_shape(hq, hkv, d, q_dtype=io, kv_dtype=kind, out_dtype=io, softmax_scale=d ** -0.5)
        dev = "cuda"
        scales = [None, None]
        if kind == "fp4":
            pools = [torch.zeros(POOL, hkv * aug.MXFP4_CELL_BYTES, dtype=torch.uint8, device=dev) for _ in range(2)]
        elif kind == "fp8":
            pools = [torch.zeros(POOL, hkv, 16, d, dtype=torch.uint8, device=dev) for _ in range(2)]
            scales = [torch.zeros(POOL, hkv, device=dev) for _ in range(2)]
        else:
            pools = [torch.zeros(POOL, hkv, 16, d, dtype=self.dtype, device=dev) for _ in range(2)]
        self.kv = rt.PagedKV(self.shape, *pools, *scales, staging_bytes=1)
        free = list(range(POOL))
        random.Random(3).shuffle(free)
        self.state = steps.State([[] for _ in range(REQS)], free)
        self.t = rt.StepTables(REQS, ROWS, WIDTH, POOL, max_draft=DRAFTS, free_ids=torch.tensor(free, dtype=torch.int32, device=dev))
        self.att = rt.TreeAttention(self.shape, self.kv, self.t)
        self.rope = rt.Rope(d, base=BASE)
        gen = torch.Generator(device=dev).manual_seed(5)
        rnd = lambda *s, std=1.0: torch.randn(*s, generator=gen, device=dev) * std  # noqa: E731
        self.eq, self.ek, self.ev = (rnd(VOCAB, h, d).to(self.dtype) for h in (hq, hkv, hkv))
        self.w = rnd(hq * d, VOCAB, std=2.0 / (hq * d) ** 0.5)
        ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
        self.ctx, self.q_len, self.parents, self.drafts, self.root = ints(REQS), ints(REQS), ints(ROWS), ints(ROWS), ints(REQS)
        self.uniform = torch.zeros(ROWS, device=dev)
        full = lambda v, t=torch.float32: torch.full((ROWS,), v, dtype=t, device=dev)  # noqa: E731
        self.setting = dict(temperature=full(0.8), top_k=full(5, torch.int32), top_p=full(0.95), min_p=full(0.02))
        self.out, self.q_rot = torch.zeros(ROWS, hq, d, dtype=self.dtype, device=dev), torch.zeros(ROWS, hq, d, dtype=self.dtype, device=dev)
        self.new = [torch.zeros(ROWS, hkv, d, dtype=self.dtype, device=dev) for _ in range(2)]
        self.tokens, self.probs = ints(ROWS), torch.zeros(ROWS, device=dev)
        self.logits, self.used = torch.zeros(ROWS, VOCAB, device=dev), ints(ROWS).long()
        self.count = ints(REQS)
        self.held = [x.clone() for x in (*pools, *scales) if x is not None]      # the cache behind the append

    def step(self):
        """One step; every tensor that it writes stands still, so that a graph can hold it."""
        from paper_2512_04013_amd import runtime as rt
        t, i = self.t, torch.arange(DRAFTS, device="cuda")
        t.update(self.ctx, self.q_len, self.parents)
        self.att.plan()
        # a request's first row is the token that it sampled last
        used = torch.cat([self.drafts, self.root]).long()
        first = torch.where(self.q_len > 0, t.q_start[:-1], ROWS + torch.arange(REQS, device="cuda"))
        used.scatter_(0, first.long(), self.root.long())
        self.used.copy_(used[:ROWS])
        self.kv.append_rows(t.slots, self.ek[self.used], self.ev[self.used], q=self.eq[self.used], rope=self.rope, positions=t.positions,
                            q_out=self.q_rot, live_rows=t.live_rows)
        self.kv.read(t.slots, *self.new)
        for a, b in zip(self.held, (self.kv.k_cache, self.kv.v_cache, self.kv.k_scale, self.kv.v_scale)):
            a.copy_(b)
        self.att.run(self.q_rot, out=self.out)
        self.logits.copy_(self.out.reshape(ROWS, -1).float() @ self.w)
        rt.sample(self.logits, self.uniform, **self.setting, tokens=self.tokens, probs=self.probs)
        # the path from the first row along drafts that are what was sampled before them
        row = (t.q_start[:-1, None] + i).clamp(max=ROWS - 1).long()
        ok = (i < self.q_len[:, None]) & (t.state == steps.OK)[:, None]
        parent, token, drawn = self.parents[row], self.used[row].int(), self.tokens[row]
        at = torch.zeros(REQS, 1, dtype=torch.int64, device="cuda")
        path, alive = [torch.where(ok[:, :1], at, -1)], ok[:, :1]
        for _ in range(DRAFTS - 1):
            fits = ok & (i > 0) & (parent == at) & (token == drawn.gather(1, at)) & alive
            alive = fits.any(1, keepdim=True)
            at = torch.where(alive, fits.int().argmax(1, keepdim=True), at)
            path.append(torch.where(alive, at, -1))
        path = torch.cat(path, 1)
        kept = path >= 0
        # its rows go behind the tokens before
        source = torch.where(kept, t.slots[row.gather(1, path.clamp(min=0))], -1).flatten()
        target = torch.where(kept, t.slots[row], -1).flatten()
        self.kv.append_rows(target, *self.kv.read(source))
        self.count.copy_(kept.sum(1))
        self.ctx.add_(self.count)
        self.root.copy_(torch.where(ok[:, :1], drawn.gather(1, at), self.root[:, None]).flatten())

    def rows(self, pools, slots):
        """K and V of slots; of fp8 caches code * scale as it is (read() rounds it to bf16)."""
        slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
        if self.kind != "fp8":
            return [f64(x) for x in self.kv.read(slots)]
        block, at = slots // 16, slots % 16
        return [f64(x.view(torch.float8_e4m3fn)[block, :, at].double() * s[block][:, :, None].double()) for x, s in zip(pools[:2], pools[2:])]

    def read(self, r, n, pools=None):
        table = self.state.table[r]
        return self.rows(pools or (self.kv.k_cache, self.kv.v_cache, self.kv.k_scale, self.kv.v_scale),
                         [table[j // 16] * 16 + j % 16 for j in range(n)])

    def check(self, ctx, q_len, parents, before):
        t, w = self.t, orope.frequencies(self.d, BASE)
        rows = sum(q_len)
        want = steps.update(self.state, ctx, q_len, parents, ROWS, WIDTH, DRAFTS)
        for name in ("q_start", "kv_len", "state"):
            assert getattr(t, name).tolist() == want[name], name
        for name in ("positions", "slots", "seen"):
            assert getattr(t, name)[:rows].tolist() == want[name], name
        # rows that were appended, as the cache gives them back
        used, positions = self.used[:rows].cpu().numpy(), np.array(want["positions"])
        live = np.array(want["slots"]) >= 0
        half = self.d // 2
        for got, x, what in ((self.q_rot, self.eq, "q"), (self.new[0], self.ek, "k")):
            if not live.any() or (what == "k" and self.kind in ("fp8", "fp4")):
                continue
            x = f64(x)[used]
            to = orope.rotate(x, positions, w)
            size = np.abs(x) + np.abs(np.roll(x, half, -1))
            within(f64(got[:rows])[live], to[live], (2.0 ** -22 * size + torch.finfo(self.dtype).eps / 2 * np.abs(to) + 1e-30)[live], what)
        if self.kind in ("f32", "bf16"):
            assert np.array_equal(f64(self.new[1][:rows])[live], f64(self.ev)[used][live])
        # attention over what the cache held
        q, out = f64(self.q_rot), f64(self.out)
        k_new, v_new = (f64(x)[:rows] for x in self.new)
        fine, g = self.kind == "f32", self.hq // self.hkv
        tokens, uniform, logits = self.tokens.tolist(), f64(self.uniform), f64(self.logits)
        for r in range(REQS):
            q0, n = want["q_start"][r], q_len[r]
            if want["state"][r] != steps.OK:
                assert not out[q0:q0 + n].any() and int(self.count[r]) == 0
                continue
            k, v = (np.concatenate([a, b[q0:q0 + n]]) for a, b in zip(before[r], (k_new, v_new)))
            if self.kind == "fp8":                     # new rows may have made a block's scale grow, its codes were rounded again
                k, v = self.read(r, ctx[r] + n, self.held)
            seen = otree.sees([m % (1 << 64) for m in want["seen"][q0:q0 + n]], ctx[r], n)
            for h in range(self.hq if n else 0):
                p = otree.weights(q[q0:q0 + n, h], k[:, h // g], seen, self.shape.softmax_scale)
                o, vh = p @ v[:, h // g], np.abs(v[:, h // g])
                size = (np.abs(q[q0:q0 + n, h]) @ np.abs(k[:, h // g]).T).max(1, initial=0.0) * self.shape.softmax_scale
                rel = 2.0 ** -24 * (self.d * size + 32 * (1 + size) + len(k)) + (0.0 if fine else 2.0 ** -8)
                bound = (1.01 * rel)[:, None] * (p @ vh + np.abs(o)) + (2.0 ** -24 if fine else 2.0 ** -8) * np.abs(o) + 1e-30
                within(out[q0:q0 + n, h], o, bound, f"request {r} head {h}")
            for i in range(q0, q0 + n):
                token, _, margin = sampling.draw(logits[i], uniform[i], temperature=float(np.float32(0.8)), top_k=5,
                                                 top_p=float(np.float32(0.95)), min_p=float(np.float32(0.02)))
                assert tokens[i] == token or margin < 1e-9, (r, i)
            # the path, and where its rows are now
            path, at = [0] if n else [], 0
            while path:
                to = [i for i in range(1, n) if parents[q0 + i] == at and used[q0 + i] == tokens[q0 + at]]
                if not to:
                    break
                at = to[0]
                path.append(at)
            assert int(self.count[r]) == len(path) and int(self.ctx[r]) == ctx[r] + len(path)
            if n:
                assert int(self.root[r]) == tokens[q0 + at]
            if self.kind != "fp8":
                for a, b, x in zip(self.read(r, ctx[r] + len(path)), before[r], (k_new, v_new)):
                    assert np.array_equal(a, np.concatenate([b, x[q0:q0 + n][path]])), r
        return [int(c) for c in self.ctx], [int(c) for c in self.count]


@pytest.mark.parametrize("kind", list(LAYERS))
def test_steps(kind):
    loop = Loop(kind)
    rng = random.Random(9)
    say(f"[drafted steps] {kind}")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ctx, graph, moved, refused = [0] * REQS, None, 0, 0
    for k in range(40):
        # a request in twenty ends, the others go on (also where they were refused)
        for r in range(REQS):
            if rng.random() < 0.05 or ctx[r] + DRAFTS > 16 * WIDTH:
                ctx[r] = 0
        q_len = [rng.choice([0, 1, DRAFTS, DRAFTS, rng.randint(1, DRAFTS)]) if k % 7 or r else 0 for r in range(REQS)]
        q_len = [1 if c and not n else n for c, n in zip(ctx, q_len)]      # (no rows and no tokens: the request gives its blocks back)
        parents = [p for n in q_len for p in [-1] + [rng.randint(0, i - 1) for i in range(1, n)] if n]
        loop.ctx.copy_(i32(ctx))
        loop.q_len.copy_(i32(q_len))
        loop.parents.copy_(i32(parents + [-1] * (ROWS - len(parents))))
        loop.drafts.copy_(i32([rng.randrange(VOCAB) for _ in range(ROWS)]))
        loop.uniform.copy_(torch.tensor([rng.random() for _ in range(ROWS)], device="cuda"))
        before = [loop.read(r, c) for r, c in enumerate(ctx)]
        torch.cuda.synchronize()
        if k < 2:
            loop.step()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    loop.step()
            graph.replay()
        torch.cuda.synchronize()
        ctx, count = loop.check(ctx, q_len, parents, before)
        moved += sum(c > 1 for c in count)
        refused += sum(s == steps.NO_BLOCKS for s in loop.t.state.tolist())
    say(f"  {moved} paths beyond the first row, {refused} refusals")
    assert moved >= 10 and refused >= 1
