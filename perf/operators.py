"""The 4-bit cache, the rows read back from a cache, and attention with score
modifiers: the passes whose speed is followed, their plain forms and exact
results.

Kinds of pass:

* ``append``: a step's new K/V rows written into a 4-bit cache (quantised there)
  and the same rows read back, as a request's are when it leaves for another
  cache format;
* ``read``: whole requests read out of a paged cache of any format;
* ``attend``: attention of a planned mixed batch, over the 4-bit cache or, with
  a cap on the scores, a bias by distance or a mask, over any cache.

Lengths and masks come from a case alone; data, block placement and queries
come from the seed. Keys and values are N(0, 1); queries N(0, std^2), so scaled
scores have the standard deviation ``std``: 1 as elsewhere in the benchmarks, 4
and more where a cap is set, which is there for scores that grow large.

A 4-bit pool is uint8 [blocks][68 * 16 * kv heads]: the codes of all heads, 1024
bytes each, then their scales, 64 bytes each. A group of 32 dims of one token
has one scale, a power of two (its exponent + 127 as a byte); a code is sign,
then the index into 0, 0.5, 1, 1.5, 2, 3, 4, 6. K: codes [16 tokens][128 dims],
the even dim in the low nibble; scales [16 tokens][4 groups]. V: codes [4 token
quads][16 dim octets][4 tokens][8 dims], scales [4 groups][16 tokens].
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
DEVICE = "cuda"
CELL = 1088            # bytes of one (block, KV head) of a 4-bit pool: 1024 of codes, 64 of scales

# (query heads, KV heads, head_dim, KV format)
LAYERS = {
    "f32-4x4-d64": (4, 4, 64, "f32"),
    "f32-8x2-d128": (8, 2, 128, "f32"),
    "bf16-16x8-d64": (16, 8, 64, "bf16"),
    "bf16-16x4-d64": (16, 4, 64, "bf16"),
    "bf16-32x8-d128": (32, 8, 128, "bf16"),
    "bf16-64x8-d128": (64, 8, 128, "bf16"),
    "fp8-32x8-d128": (32, 8, 128, "fp8"),
    "fp8-64x8-d128": (64, 8, 128, "fp8"),
    "fp4-8x8-d128": (8, 8, 128, "fp4"),
    "fp4-16x8-d128": (16, 8, 128, "fp4"),
    "fp4-32x8-d128": (32, 8, 128, "fp4"),
    "fp4-64x8-d128": (64, 8, 128, "fp4"),
}

# decodes: contexts lognormal around "ctx" (sigma 0.8, capped) or uniform from "ctx" to "cap"; chunks of "rows"
# rows over up to "prior" earlier tokens. "span": window length, or mean length of a prefix or document.
_BASE = {"decodes": 0, "ctx": 1, "cap": 1, "dist": "lognormal", "chunks": 0, "rows": 1, "prior": 0, "lengths": 0,
         "softcap": 0.0, "slopes": False, "mask": "causal", "span": 0, "std": 1.0}


def _case(**kw):
    return {**_BASE, **kw}


def listed():
    return [
        # a decode step of a lightly loaded server: latency of two small launches
        _case(name="append4-decode-8b", kind="append", layer="fp4-32x8-d128", decodes=64, ctx=1200, cap=8192),
        # the rows of an 8192-token budget, whole blocks and ragged ends
        _case(name="append4-prefill-64x8", kind="append", layer="fp4-64x8-d128", decodes=31, ctx=800, cap=8192, chunks=15, rows=541, prior=2048),
        # 16 paused requests leave an fp8 cache for another format
        _case(name="read-fp8-64x8", kind="read", layer="fp8-64x8-d128", decodes=16, ctx=1500, cap=8192),
        # the smallest mixed batch
        _case(name="attend4-tiny", kind="attend", layer="fp4-16x8-d128", decodes=6, ctx=16, cap=256, dist="uniform", chunks=1, rows=33, prior=64),
        # decodes at full concurrency, eight query heads per KV head
        _case(name="attend4-decode-64x8", kind="attend", layer="fp4-64x8-d128", decodes=512, ctx=2500, cap=16384),
        # retrieval-augmented prompts: 64 decodes over 16k to 32k keys
        _case(name="attend4-long-8b", kind="attend", layer="fp4-32x8-d128", decodes=64, ctx=16384, cap=32768, dist="uniform"),
        # prefill-dominated batch of an 8192-token budget
        _case(name="attend4-prefill-64x8", kind="attend", layer="fp4-64x8-d128", chunks=16, rows=512, prior=2048),
        # decodes with capped scores in a layer of local attention
        _case(name="window-cap-decode-8b", kind="attend", layer="bf16-32x8-d128", decodes=256, ctx=4000, cap=16384, softcap=50.0, mask="window", span=1024, std=6.0),
        # packed documents, some of them padding, biased by distance, in long chunks
        _case(name="documents-alibi-prefill-8b", kind="attend", layer="bf16-32x8-d128", chunks=2, rows=4096, prior=2048, slopes=True, mask="documents", span=900),
        # prompts attended from both sides, capped scores, over the fp8 cache, beside decodes
        _case(name="prefix-cap-fp8-64x8", kind="attend", layer="fp8-64x8-d128", decodes=64, ctx=2000, cap=8192, chunks=8, rows=512, prior=1024, softcap=30.0, mask="prefix", span=700, std=4.0),
        # everything at once over the 4-bit cache: capped, biased, windowed, chunks and decodes
        _case(name="all-fp4-8b", kind="attend", layer="fp4-32x8-d128", decodes=128, ctx=3000, cap=16384, chunks=3, rows=333, prior=4096, softcap=30.0, slopes=True, mask="window", span=2048, std=4.0),
        # the same in fp32, at the smallest size
        _case(name="all-tiny-f32", kind="attend", layer="f32-4x4-d64", decodes=6, ctx=16, cap=256, dist="uniform", chunks=2, rows=32, prior=64, softcap=20.0, slopes=True, mask="documents", span=40, std=4.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the listed kinds over their ranges, odd sizes included."""
    kind = rng.choice(["append", "read", "four", "four", "four", "scored", "scored", "scored"])
    seed = rng.randrange(1, 1 << 20)
    fp4 = sorted(k for k in LAYERS if k.startswith("fp4"))
    if kind == "append":
        return _case(kind="append", layer=rng.choice(fp4), decodes=_log_int(rng, 1, 256), ctx=_log_int(rng, 16, 2000), cap=8192,
                     chunks=rng.choice([0, 1, 4, 8]), rows=_log_int(rng, 2, 600), prior=rng.choice([0, 512, 2048]), lengths=seed)
    if kind == "read":
        return _case(kind="read", layer=rng.choice(sorted(LAYERS)), decodes=_log_int(rng, 1, 16), ctx=_log_int(rng, 16, 1500), cap=8192, lengths=seed)
    layer = rng.choice(fp4 if kind == "four" else sorted(LAYERS))
    small = layer.startswith("f32")          # fp32 is the small, exact configuration
    n = _log_int(rng, 1, 64 if small else 400)
    ctx = _log_int(rng, 16, max(64, min(512 if small else 20_000, (20_000 if small else 800_000) // (2 * n))))
    c = _case(kind="attend", layer=layer, decodes=n, ctx=ctx, cap=min(32768, 6 * ctx), lengths=seed)
    if rng.random() < 0.6:
        rows = _log_int(rng, 2, 48 if small else 2048)
        c.update(chunks=rng.randint(1, max(1, min(8, 4096 // rows))), rows=rows, prior=rng.choice([0, 64, 256] if small else [0, 512, 4096]))
        if rng.random() < 0.3:
            c.update(decodes=0)
    if kind == "scored":
        c.update(softcap=rng.choice([0.0, 20.0, 30.0, 50.0]), slopes=rng.random() < 0.4, mask=rng.choice(["causal", "window", "prefix", "documents"]),
                 span=_log_int(rng, 16, 256 if small else 4096))
        c["std"] = rng.choice([4.0, 6.0]) if c["softcap"] else 1.0
        if not c["softcap"] and not c["slopes"] and c["mask"] == "causal":
            c["slopes"] = True
    return c


def _lengths(case):
    """(query rows, context) of each request: chunks first, then decodes. A read takes whole contexts."""
    rng = random.Random(case["lengths"])
    out = []
    for i in range(case["chunks"]):
        prior = rng.randint(0, case["prior"])
        rows = case["rows"]
        if case["lengths"] and i == case["chunks"] - 1 and rows > 2:
            rows = rng.randint(2, rows)      # a prompt ends where it does
        out.append((rows, rows + prior))
    for _ in range(case["decodes"]):
        if case["dist"] == "uniform":
            ctx = rng.randint(case["ctx"], case["cap"])
        else:
            ctx = min(case["cap"], max(1, round(rng.lognormvariate(math.log(case["ctx"]), 0.8))))
        out.append((ctx if case["kind"] == "read" else 1, ctx))
    return out


def _seen(case, pairs):
    """First key and one past the last key of every query row, in row order."""
    rng = random.Random(case["lengths"] + 1)
    first, end = [], []
    for n, ctx in pairs:
        pos = np.arange(ctx - n, ctx, dtype=np.int64)
        lo, hi = np.zeros(n, np.int64), pos + 1
        if case["mask"] == "window":
            lo = np.maximum(0, pos - case["span"] + 1)
        elif case["mask"] == "prefix":
            hi = np.maximum(hi, min(ctx, rng.randint(0, 2 * case["span"])))
        elif case["mask"] == "documents":
            starts, pad, at = [], [], 0
            while at < ctx:
                starts.append(at)
                pad.append(rng.random() < 0.06 and at > 0)     # padding between documents: its rows see nothing
                at += rng.randint(1, 2 * case["span"])
            doc = np.searchsorted(np.array(starts), pos, side="right") - 1
            lo = np.array(starts)[doc]
            hi = np.where(np.array(pad)[doc], lo, hi)
        first.append(lo)
        end.append(hi)
    return np.concatenate(first), np.concatenate(end)


def _slopes(hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEVICE)


# ---- the 4-bit format, in 32-bit torch ---------------------------------------------------

_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_BOUNDS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)    # midpoints: a tie goes to the even index


def _quantise4(x):
    """x [..., 128] float32 -> codes [..., 128] and scale bytes [..., 4], uint8."""
    g = x.unflatten(-1, (4, 32))
    a = g.abs().amax(-1)
    bits = (a.view(torch.int32) + (1 << 21)) >> 23       # exponent field, one more from 1.75 * 2^k on
    byte = (bits - 2).clamp(2, 252)
    y = torch.ldexp(g, (127 - byte)[..., None])
    m = y.abs()
    code = torch.zeros_like(m, dtype=torch.uint8)
    for i, b in enumerate(_BOUNDS):
        code += ((m > b) if i % 2 == 0 else (m >= b)).to(torch.uint8)
    return (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2), byte.to(torch.uint8)


def _values4(codes, scales):
    """codes [..., 128] and scale bytes [..., 4] -> float32 [..., 128]."""
    level = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), dtype=torch.float32, device=codes.device)
    return torch.ldexp(level[codes.int()].unflatten(-1, (4, 32)), (scales.int() - 127)[..., None]).flatten(-2)


def _pack4(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack4(byte):
    return torch.stack((byte & 15, byte >> 4), -1).flatten(-2)


def _views4(pool, hkv, is_v):
    """Views of a 4-bit pool's codes and scales, by (block, head, token ...)."""
    codes, scales = pool[:, :hkv * 1024], pool[:, hkv * 1024:]
    if is_v:
        return codes.view(-1, hkv, 4, 16, 4, 4), scales.view(-1, hkv, 4, 16)
    return codes.view(-1, hkv, 16, 64), scales.view(-1, hkv, 16, 4)


def _load4(pool, hkv, is_v, blk, slot):
    """Rows at (blk, slot) of a 4-bit pool: float32 [n, hkv, 128]."""
    codes, scales = _views4(pool, hkv, is_v)
    if is_v:
        c = codes[blk, :, slot // 4, :, slot % 4]          # [n, hkv, 16 octets, 4 bytes]
        return _values4(_unpack4(c.flatten(-2)), scales[blk, :, :, slot])
    return _values4(_unpack4(codes[blk, :, slot]), scales[blk, :, slot])


def _store4(pool, hkv, is_v, blk, slot, x):
    """Rows x [n, hkv, 128] (float32) into a 4-bit pool at (blk, slot)."""
    codes, scales = _views4(pool, hkv, is_v)
    c, s = _quantise4(x)
    c = _pack4(c)
    if is_v:
        codes[blk, :, slot // 4, :, slot % 4] = c.unflatten(-1, (16, 4))
        scales[blk, :, :, slot] = s
    else:
        codes[blk, :, slot] = c
        scales[blk, :, slot] = s


# ---- inputs ---------------------------------------------------------------------------------

class _Batch:
    """Lengths, masks, paged layout and data of one case."""

    def __init__(self, case, seed):
        self.hq, self.hkv, self.d, self.kv = LAYERS[case["layer"]]
        pairs = _lengths(case)
        self.q_len = np.array([q for q, _ in pairs], np.int64)
        self.ctx = np.array([c for _, c in pairs], np.int64)
        nblk = -(-self.ctx // BLOCK)
        self.bt_start = np.concatenate([[0], np.cumsum(nblk)]).astype(np.int32)
        self.q_start = np.concatenate([[0], np.cumsum(self.q_len)]).astype(np.int32)
        self.rows = int(self.q_len.sum())
        used = int(nblk.sum())
        self.pool = used + used // 4 + 64
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(seed)
        perm = torch.randperm(self.pool, generator=self.gen, device=DEVICE, dtype=torch.int64).to(torch.int32)
        self.block_ids = perm[:used].contiguous()
        self.dtype = torch.float32 if self.kv == "f32" else torch.bfloat16
        pos = np.concatenate([np.arange(c - q, c) for q, c in pairs])
        req = np.repeat(np.arange(len(pairs)), self.q_len)
        table = self.block_ids.cpu().numpy()
        self.blk = torch.from_numpy(table[self.bt_start[req] + pos // BLOCK].astype(np.int64)).to(DEVICE)
        self.slot = torch.from_numpy(pos % BLOCK).to(DEVICE)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=DEVICE, dtype=self.dtype)

    def cache(self):
        """A pool of K or V, every slot filled, and its scales (fp8)."""
        shape = (self.pool, self.hkv, BLOCK, self.d)
        if self.kv in ("f32", "bf16"):
            return self.normal(*shape), None
        step = 1 << 13
        if self.kv == "fp4":
            # codes and scales in the places of K: V's places permute equal distributions
            pool = torch.empty(self.pool, CELL * self.hkv, dtype=torch.uint8, device=DEVICE)
            codes, scales = _views4(pool, self.hkv, False)
            for b0 in range(0, self.pool, step):
                c, s = _quantise4(self.normal(min(step, self.pool - b0), *shape[1:]).float())
                codes[b0:b0 + step] = _pack4(c)
                scales[b0:b0 + step] = s
            return pool, None
        codes = torch.empty(shape, dtype=torch.uint8, device=DEVICE)
        scale = torch.empty(shape[:2], dtype=torch.float32, device=DEVICE)
        for b0 in range(0, self.pool, step):
            x = self.normal(min(step, self.pool - b0), *shape[1:]).float()
            s = (x.abs().amax(dim=(2, 3)) / 448.0).clamp_min(1e-12)
            codes[b0:b0 + step] = (x / s[:, :, None, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[b0:b0 + step] = s
        return codes, scale


def _inputs(case, seed):
    """Everything a pass reads, as plain tensors."""
    b = _Batch(case, seed)
    s = {"case": case, "b": b}
    if case["kind"] == "append":
        s["k_new"], s["v_new"] = b.normal(b.rows, b.hkv, b.d), b.normal(b.rows, b.hkv, b.d)
    if case["kind"] == "attend":
        s["q"] = (b.normal(b.rows, b.hq, b.d).float() * case["std"]).to(b.dtype)
        s["slopes"] = _slopes(b.hq) if case["slopes"] else None
    s["k"], s["k_scale"] = b.cache()
    s["v"], s["v_scale"] = b.cache()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    b = s["b"]
    s["slots"] = (b.blk * BLOCK + b.slot).contiguous()          # where each row's token lies
    if case["kind"] == "attend":
        lo, hi = _seen(case, list(zip(b.q_len.tolist(), b.ctx.tolist())))
        s["seen"] = (lo, hi)
        s["first"], s["end"] = torch.from_numpy(lo).to(DEVICE), torch.from_numpy(hi).to(DEVICE)
    if own:
        import paper_2512_04013_amd as aug
        from paper_2512_04013_amd import runtime as rt
        io = "f32" if b.kv == "f32" else "bf16"
        shape = aug.make_shape(b.hq, b.hkv, b.d, io, b.kv, io, 1.0 / math.sqrt(b.d))
        s["kv"] = rt.PagedKV(shape, s["k"], s["v"], s["k_scale"], s["v_scale"], staging_bytes=1)
        if case["kind"] != "read":
            masked = case["kind"] == "attend" and case["mask"] != "causal"
            first, end = s["seen"] if masked else (None, None)
            s["att"] = rt.MixedAttention(shape, s["kv"], b.q_start, b.ctx, b.bt_start, b.block_ids.cpu().numpy(), b.block_ids,
                                         row_first=first, row_end=end)
        s["rows"] = [torch.empty(b.rows, b.hkv, b.d, dtype=b.dtype, device=DEVICE) for _ in range(2)]
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        if case["kind"] == "attend":
            return state["att"].run(state["q"], softcap=case["softcap"], slopes=state["slopes"])
        if case["kind"] == "append":
            state["att"].append(state["k_new"], state["v_new"])
        return state["kv"].read(state["slots"], *state["rows"])
    if case["kind"] == "attend":
        return _plain_attention(state)
    b = state["b"]
    if case["kind"] == "append":
        _store4(state["k"], b.hkv, False, b.blk, b.slot, state["k_new"].float())
        _store4(state["v"], b.hkv, True, b.blk, b.slot, state["v_new"].float())
    slots = state["slots"]
    return tuple(_plain_rows(state, name, slots // BLOCK, slots % BLOCK).to(b.dtype) for name in ("k", "v"))


def _plain_rows(state, name, blk, slot):
    """Rows of the K or V cache at (blk, slot): float32 [n, hkv, d]."""
    b, pool = state["b"], state[name]
    if b.kv == "fp4":
        return _load4(pool, b.hkv, name == "v", blk, slot)
    x = pool[blk, :, slot]
    if b.kv == "fp8":
        return x.view(torch.float8_e4m3fn).float() * state[name + "_scale"][blk][:, :, None]
    return x.float()


def _scored(state, s, pos, key, first, end):
    """Scores s [..., hkv, rows, g, keys] (already scaled) capped, biased and masked; the other arguments are
    positions that broadcast to [..., rows, keys]."""
    case, b = state["case"], state["b"]
    if case["softcap"]:
        s = torch.tanh(s.div_(case["softcap"])).mul_(case["softcap"])
    if state["slopes"] is not None:
        s -= state["slopes"].view(b.hkv, 1, -1, 1) * (pos - key).abs().float()[..., None, :, None, :]
    return s.masked_fill_(((key < first) | (key >= end))[..., None, :, None, :], -math.inf)


def _plain_attention(state):
    """softmax(modified scores) V in 32 bits: the chunks one after another, all decodes at once, block by block."""
    b, case = state["b"], state["case"]
    g, scale = b.hq // b.hkv, 1.0 / math.sqrt(b.d)
    out = torch.empty(b.rows, b.hq, b.d, dtype=b.dtype, device=DEVICE)
    q, ids, slot = state["q"], b.block_ids.long(), torch.arange(BLOCK, device=DEVICE)
    chunks = case["chunks"]
    for r, (n, ctx) in enumerate(zip(b.q_len[:chunks].tolist(), b.ctx[:chunks].tolist())):
        rows = slice(int(b.q_start[r]), int(b.q_start[r + 1]))
        key = torch.arange(ctx, device=DEVICE)
        blk = ids[int(b.bt_start[r]) + key // BLOCK]
        k = _plain_rows(state, "k", blk, key % BLOCK).permute(1, 2, 0).contiguous()       # [hkv, d, ctx]
        v = _plain_rows(state, "v", blk, key % BLOCK).transpose(0, 1).contiguous()        # [hkv, ctx, d]
        x = q[rows].float().view(n, b.hkv, g, b.d).transpose(0, 1).reshape(b.hkv, n * g, b.d)
        s = torch.bmm(x, k).mul_(scale).view(b.hkv, n, g, ctx)
        s = _scored(state, s, torch.arange(ctx - n, ctx, device=DEVICE)[:, None], key[None, :], state["first"][rows, None], state["end"][rows, None])
        p = torch.exp(s.sub_(s.amax(-1, keepdim=True).clamp_min(-3e38)))
        total = p.sum(-1, keepdim=True)
        p /= torch.where(total == 0, 1.0, total)
        o = torch.bmm(p.view(b.hkv, n * g, ctx), v)
        out[rows] = o.view(b.hkv, n, g, b.d).transpose(0, 1).reshape(n, b.hq, b.d).to(b.dtype)
    count = len(b.ctx) - chunks
    if count == 0:
        return out
    nblk = torch.from_numpy(np.diff(b.bt_start[chunks:]).astype(np.int64)).to(DEVICE)
    ids = ids[int(b.bt_start[chunks]):]
    req = torch.repeat_interleave(torch.arange(count, device=DEVICE), nblk)              # each block's request
    key = ((torch.arange(len(ids), device=DEVICE) - (nblk.cumsum(0) - nblk)[req]) * BLOCK)[:, None] + slot
    rows = slice(int(b.q_start[chunks]), b.rows)
    pos = torch.from_numpy(b.ctx[chunks:] - 1).to(DEVICE)
    blk, slots = ids.repeat_interleave(BLOCK), slot.repeat(len(ids))
    layout = (len(ids), BLOCK, b.hkv, b.d)
    k = _plain_rows(state, "k", blk, slots).view(layout).permute(0, 2, 3, 1).reshape(-1, b.d, BLOCK)
    x = q[rows].float().view(count, b.hkv, g, b.d)[req].view(-1, g, b.d)
    s = torch.bmm(x, k).mul_(scale).view(len(ids), b.hkv, 1, g, BLOCK)
    s = _scored(state, s, pos[req, None, None], key[:, None, :], state["first"][rows][req, None, None],
                torch.minimum(state["end"][rows], pos + 1)[req, None, None]).squeeze(2)
    top = torch.full((count, b.hkv, g), -3e38, device=DEVICE).index_reduce_(0, req, s.amax(-1), "amax")
    p = torch.exp(s.sub_(top[req][..., None]))
    total = torch.zeros(count, b.hkv, g, device=DEVICE).index_add_(0, req, p.sum(-1))
    v = _plain_rows(state, "v", blk, slots).view(layout).transpose(1, 2).reshape(-1, BLOCK, b.d)
    part = torch.bmm(p.view(-1, g, BLOCK), v).view(len(ids), b.hkv, g, b.d)
    o = torch.zeros(count, b.hkv, g, b.d, device=DEVICE).index_add_(0, req, part)
    out[rows] = (o / torch.where(total == 0, 1.0, total)[..., None]).view(count, b.hq, b.d).to(b.dtype)
    return out


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    hq, hkv, d, kv = LAYERS[case["layer"]]
    io = 4 if kv == "f32" else 2
    row = {"f32": 4 * d, "bf16": 2 * d, "fp8": d, "fp4": 68}[kv]        # bytes of one cached row of K or V
    pairs = _lengths(case)
    rows = sum(q for q, _ in pairs)
    if case["kind"] != "attend":
        b = rows * hkv * 2 * (row + io * d) + rows * 8                   # read: the cache, the slots, the rows
        b += rows * hkv * 2 * (row + io * d) if case["kind"] == "append" else 0
        return {"bytes": b, "flops": 0}
    lo, hi = _seen(case, pairs)
    keys, at = 0, 0
    for q, ctx in pairs:                                                  # keys that some row of the request sees
        a, e = lo[at:at + q], hi[at:at + q]
        step = np.zeros(ctx + 1, np.int64)
        live = e > a
        np.add.at(step, a[live], 1)
        np.add.at(step, e[live], -1)
        keys += int(np.count_nonzero(np.cumsum(step)[:ctx]))
        at += q
    b = keys * hkv * 2 * row + (keys // BLOCK) * (4 + (8 * hkv if kv == "fp8" else 0)) + rows * hq * d * 2 * io
    return {"bytes": b, "flops": 4 * d * hq * int(np.maximum(hi - lo, 0).sum())}


# ---- exact results ----------------------------------------------------------------------------------

def _cell4(pool, hkv, ids, is_v):
    """Blocks ids of a 4-bit pool, decoded field by field: float64 [n blocks, hkv, 16, 128]."""
    raw = pool[ids]
    codes = raw[:, :1024 * hkv].reshape(len(ids), hkv, 1024).long()
    power = raw[:, 1024 * hkv:].reshape(len(ids), hkv, 64).double() - 127.0
    nib = torch.empty(len(ids), hkv, 2048, dtype=torch.int64, device=raw.device)
    nib[..., 0::2], nib[..., 1::2] = codes % 16, codes // 16
    field, mant = (nib % 8) // 2, nib % 2
    mag = torch.where(field == 0, 0.5 * mant.double(), (1.0 + 0.5 * mant.double()) * 2.0 ** (field.double() - 1.0))
    val = torch.where(nib >= 8, -mag, mag)
    if is_v:
        val = val.reshape(-1, hkv, 4, 16, 4, 8).permute(0, 1, 2, 4, 3, 5).reshape(-1, hkv, 16, 128)
        power = power.reshape(-1, hkv, 4, 16).transpose(2, 3)
    else:
        val, power = val.reshape(-1, hkv, 16, 128), power.reshape(-1, hkv, 16, 4)
    return val * torch.repeat_interleave(2.0 ** power, 32, dim=-1)


def _blocks64(s, ids, name):
    b, pool = s["b"], s[name]
    if b.kv == "fp4":
        return _cell4(pool, b.hkv, ids, name == "v")
    x = pool[ids]
    if b.kv == "fp8":
        return x.view(torch.float8_e4m3fn).double() * s[name + "_scale"][ids].double()[:, :, None, None]
    return x.double()


def _nearest4(x):
    """The 4-bit cache's value of every element of x [n, hkv, 128], float64: each group's power of two from the
    logarithm of its largest magnitude, each element the nearest multiple (the even code between two)."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    for g in range(4):
        y = x[..., 32 * g:32 * g + 32].double()
        a = y.abs().max(-1, keepdim=True).values
        frac, e = torch.frexp(a)                              # a = frac * 2^e, frac in [0.5, 1)
        e = torch.where(frac >= 0.875, e, e - 1)
        scale = 2.0 ** (torch.where(a > 0, e.double(), torch.full_like(a, -200.0)) - 2.0).clamp(-125.0, 125.0)
        gap = (y.abs() / scale).unsqueeze(-1) - level
        gap = gap.abs() + torch.tensor([0.0, 1e-12] * 4, dtype=torch.float64, device=x.device)     # even codes win ties
        out[..., 32 * g:32 * g + 32] = torch.copysign(level[gap.argmin(-1)] * scale, y)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    b = s["b"]
    if case["kind"] == "append":
        return _nearest4(s["k_new"]), _nearest4(s["v_new"])
    if case["kind"] == "read":
        got = []
        for name in ("k", "v"):
            rows = []
            for r, ctx in enumerate(b.ctx.tolist()):
                x = _blocks64(s, b.block_ids[int(b.bt_start[r]):int(b.bt_start[r + 1])].long(), name)
                rows.append(x.transpose(1, 2).reshape(-1, b.hkv, b.d)[:ctx])
            got.append(torch.cat(rows))
        return tuple(got)
    lo, hi = _seen(case, list(zip(b.q_len.tolist(), b.ctx.tolist())))
    g = b.hq // b.hkv
    out = torch.zeros(b.rows, b.hq, b.d, dtype=torch.float64, device=DEVICE)
    for r in range(len(b.ctx)):
        q0, q1, ctx = int(b.q_start[r]), int(b.q_start[r + 1]), int(b.ctx[r])
        ids = b.block_ids[int(b.bt_start[r]):int(b.bt_start[r + 1])].long()
        kk, vv = _blocks64(s, ids, "k"), _blocks64(s, ids, "v")
        j = torch.arange(ctx, dtype=torch.float64, device=DEVICE)
        i = torch.arange(ctx - (q1 - q0), ctx, dtype=torch.float64, device=DEVICE)[:, None, None]
        a = torch.from_numpy(lo[q0:q1]).to(DEVICE)[:, None, None]
        e = torch.from_numpy(hi[q0:q1]).to(DEVICE)[:, None, None]
        seen = (j >= a) & (j < e)
        for h in range(b.hkv):
            k = kk[:, h].reshape(-1, b.d)[:ctx]
            v = vv[:, h].reshape(-1, b.d)[:ctx]
            x = s["q"][q0:q1, h * g:(h + 1) * g].double().reshape(-1, b.d)
            z = torch.matmul(x, k.t().contiguous()).reshape(q1 - q0, g, ctx) * b.d ** -0.5
            if case["softcap"] > 0:
                z = case["softcap"] * torch.tanh(z / case["softcap"])
            if case["slopes"]:
                z = z - s["slopes"][h * g:(h + 1) * g].double()[None, :, None] * torch.abs(i - j)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            w = torch.softmax(z, -1)
            w = torch.where(seen.any(-1, keepdim=True), w, torch.zeros_like(w))
            out[q0:q1, h * g:(h + 1) * g] = torch.matmul(w.reshape(-1, ctx), v).reshape(q1 - q0, g, b.d)
    return out
