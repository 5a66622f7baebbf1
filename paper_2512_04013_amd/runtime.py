"""Device-side plumbing around the C ABI: torch tensors for the pool, the
plan image and the workspace, and one call per step of the hot path.

Everything here is argument marshalling and memory management (torch owns
the device memory and the stream); the arithmetic runs in libaug.so.
"""

from __future__ import annotations

import contextlib
import time

import numpy as np
import torch

from . import (AUG_BF16, AUG_F32, AUG_MXFP4, MAX_DRAFT, MXFP4_CELL_BYTES, STEP_SCRATCH_BYTES, _current_stream, aug_attn_mixed, aug_attn_plan,
               aug_attn_tree, aug_kv_append, aug_kv_park, aug_kv_read, aug_kv_record_bytes, aug_kv_resume, aug_plan_upload,
               aug_rope_append, aug_rope_init, aug_rope_rows, aug_sample, aug_sample_args, aug_step_tables, aug_step_tables_args, aug_tree_batch, aug_tree_plan,
               aug_tree_plan_size, make_shape)

_TORCH_STORAGE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8, "fp4": torch.uint8}


def to_device_array(x: np.ndarray, dtype: str, device) -> torch.Tensor:
    """Host bit patterns (float32 / uint16 bf16 / uint8 fp8 and 4-bit pools) -> device tensor."""
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).view(torch.bfloat16).to(device)
    if dtype in ("fp8", "fp4"):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.uint8)).to(device)
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(device)


def to_host_f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().float().cpu().numpy().astype(np.float64)


def _allocating_on(stream, device):
    """Context in which torch allocates from ``stream`` (a torch stream, a raw
    handle, or None for the current one)."""
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _on(index: int):
    """Context in which ``index`` is torch's current device: the library's calls
    are made for the current one. Host memory (-1) is refused: no kernel reads it."""
    if index < 0:
        raise ValueError("tensors in host memory: this call needs them on a GPU")
    return contextlib.nullcontext() if torch.cuda.current_device() == index else torch.cuda.device(index)


def _check_rows(t, name, rows, heads, dim, dtype, index):
    """Rows [rows][heads][dim] on a device whose heads lie together (rows may lie further apart)."""
    if t.shape != (rows, heads, dim) or t.dtype != dtype or t.get_device() != index or t.stride(2) != 1 or \
            (heads > 1 and t.stride(1) != dim):
        raise ValueError(f"{name}: rows of shape ({rows}, {heads}, {dim}) and {dtype} on device {index}, heads of a row together, "
                         f"got {t.dtype} {tuple(t.shape)}, strides {t.stride()} on {t.device}")


def _check_vector(t, name, n, dtype, index):
    if t.shape != (n,) or t.dtype != dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} vector of {n} on device {index}, got {t.dtype} {tuple(t.shape)} on {t.device}")


class PagedKV:
    """A KV pool on the device plus its park/resume staging."""

    def __init__(self, shape, k_cache, v_cache, k_scale=None, v_scale=None, staging_bytes=1 << 28):
        self.shape = shape
        self.k_cache, self.v_cache = k_cache, v_cache
        self.k_scale, self.v_scale = k_scale, v_scale
        self.num_pool_blocks = int(k_cache.shape[0])
        if shape.kv_dtype == AUG_MXFP4:
            want = (self.num_pool_blocks, shape.num_kv_heads * MXFP4_CELL_BYTES)
            for t in (k_cache, v_cache):
                if tuple(t.shape) != want or t.dtype != torch.uint8:
                    raise ValueError(f"a 4-bit pool is uint8 of shape {want}, got {t.dtype} {tuple(t.shape)}")
        # what read() gives out, and where
        self._row = (shape.num_kv_heads, shape.head_dim)
        self._row_dtype = torch.float32 if shape.kv_dtype == AUG_F32 else torch.bfloat16
        self._device = k_cache.get_device()
        self.record_bytes = aug_kv_record_bytes(shape)
        staging_bytes = max(self.record_bytes, (staging_bytes // self.record_bytes) * self.record_bytes)
        self.staging = torch.empty(staging_bytes, dtype=torch.uint8, device=k_cache.device)

    def host_buffer(self, n_blocks: int) -> torch.Tensor:
        return torch.empty(max(1, n_blocks * self.record_bytes), dtype=torch.uint8, pin_memory=True)

    def park(self, blocks_host: np.ndarray, blocks_dev: torch.Tensor, host_dst: torch.Tensor, stream=None):
        aug_kv_park(self.shape, self.k_cache, self.v_cache, self.k_scale, self.v_scale, blocks_dev,
                    len(blocks_host), self.num_pool_blocks, host_dst, self.staging,
                    block_ids_host=blocks_host, stream=stream)

    def resume(self, blocks_host: np.ndarray, blocks_dev: torch.Tensor, host_src: torch.Tensor, stream=None):
        aug_kv_resume(self.shape, self.k_cache, self.v_cache, self.k_scale, self.v_scale, blocks_dev,
                      len(blocks_host), self.num_pool_blocks, host_src, self.staging,
                      block_ids_host=blocks_host, stream=stream)

    def read(self, slots: torch.Tensor, k_out: torch.Tensor = None, v_out: torch.Tensor = None, stream=None):
        """The K and V rows ([n][H_kv][D], float32 for f32 pools, else bf16) of
        the tokens in ``slots`` (int64, block * 16 + slot): what ``append`` takes,
        so a request moves to a pool of another format. Returns (k, v). Rows that
        are allocated here belong to ``stream``, as if it were torch's current
        one: another stream waits for it before it reads them."""
        if slots.dtype != torch.int64 or slots.dim() != 1 or not slots.is_contiguous() or \
                slots.get_device() != self._device:
            raise ValueError(f"slots must be a contiguous int64 vector on {self.k_cache.device}, got {slots.dtype} "
                             f"{tuple(slots.shape)} on {slots.device}")
        n = len(slots)
        want, dtype = (n, *self._row), self._row_dtype
        if k_out is None or v_out is None:
            # on the stream that writes them: memory that the current stream gave
            # back may still be in use there
            with _allocating_on(stream, slots.device):
                k_out = torch.empty(want, dtype=dtype, device=slots.device) if k_out is None else k_out
                v_out = torch.empty(want, dtype=dtype, device=slots.device) if v_out is None else v_out
        for t in (k_out, v_out):
            if t.shape != want or t.dtype != dtype or not t.is_contiguous() or t.get_device() != self._device:
                raise ValueError(f"K/V rows must be contiguous {dtype} of shape {want} on {slots.device}, got "
                                 f"{t.dtype} {tuple(t.shape)} on {t.device}")
        aug_kv_read(self.shape, self.k_cache, self.v_cache, self.k_scale, self.v_scale, slots, n,
                    self.num_pool_blocks, k_out, v_out, stream=stream)
        return k_out, v_out


    def append_rows(self, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor = None, rope: "Rope" = None,
                    positions: torch.Tensor = None, q_out: torch.Tensor = None, live_rows: torch.Tensor = None, stream=None):
        """Write K/V rows ([n][H_kv][D], rows may be strided) into ``slots`` (int64,
        block * 16 + slot; rows of slots outside the pool are skipped), K rotated by
        ``positions`` (int32) where a ``rope`` is given. With ``q`` its rows are
        rotated too, into ``q_out`` (may be ``q``; allocated on ``stream`` if None),
        which is returned. Without a rope and with what ``read`` returns, rows move
        to other slots. In an fp8 pool, whose blocks share a scale, the rows of a block
        follow one another, and what its slots above them held is lost. ``live_rows`` (int32 [1], such as ``StepTables.live_rows``): how
        many of the rows there are; those behind are passed over."""
        n, (hkv, dim), index = len(slots), self._row, self._device
        _check_vector(slots, "slots", n, torch.int64, index)
        _check_rows(k, "k", n, hkv, dim, self._row_dtype, index)
        _check_rows(v, "v", n, hkv, dim, self._row_dtype, index)
        if live_rows is not None:
            _check_vector(live_rows, "live_rows", 1, torch.int32, index)
        if rope is None and (q is not None or positions is not None):
            raise ValueError("queries and positions need a rope")
        if rope is not None:
            if positions is None:
                raise ValueError("a rope needs positions")
            _check_vector(positions, "positions", n, torch.int32, index)
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
        else:
            hq = self.shape.num_q_heads
            _check_rows(q, "q", n, hq, dim, self._row_dtype, index)
            if q_out is None:
                with _allocating_on(stream, q.device):
                    q_out = torch.empty((n, hq, dim), dtype=q.dtype, device=q.device)
            _check_rows(q_out, "q_out", n, hq, dim, self._row_dtype, index)
        with _on(index):
            aug_rope_append(self.shape, None if rope is None else rope.angles, positions, slots, q, k, v, q_out, self.k_cache,
                            self.v_cache, self.k_scale, self.v_scale, self.num_pool_blocks, live_rows=live_rows, stream=stream)
        return q_out


class Rope:
    """Rotary positions: the angles of the first ``rotary_dim`` dims of a head, in
    halves (dims i and i + rotary_dim / 2) or ``interleaved`` (2i and 2i + 1), with
    ``scaling`` "none", "linear", "bands" or "ramp" for long contexts (the formulas
    are in aug.h)."""

    def __init__(self, rotary_dim: int, base: float = 10000.0, interleaved: bool = False, scaling="none", factor: float = 1.0,
                 low: float = 1.0, high: float = 32.0, original_len: int = 0, magnitude: float = 1.0):
        self.angles = aug_rope_init(rotary_dim, interleaved, base, scaling, factor, low, high, original_len, magnitude)


def rope_rows(shape, rope: Rope, positions: torch.Tensor, q: torch.Tensor = None, k: torch.Tensor = None, q_out: torch.Tensor = None,
              k_out: torch.Tensor = None, stream=None):
    """Rotate rows of q ([rows][H_q][D]) and k ([rows][H_kv][D]; either may be
    None, rows may be strided) by ``positions`` (int32). Outputs may be the inputs;
    those that are None are allocated on ``stream``. Returns (q_out, k_out).
    Gradients go back through the same call with negated positions."""
    n, index = len(positions), positions.get_device()
    _check_vector(positions, "positions", n, torch.int32, index)
    dtype = torch.float32 if shape.q_dtype == AUG_F32 else torch.bfloat16
    outs = []
    for name, x, out, heads in (("q", q, q_out, shape.num_q_heads), ("k", k, k_out, shape.num_kv_heads)):
        if x is not None:
            _check_rows(x, name, n, heads, shape.head_dim, dtype, index)
            if out is None:
                with _allocating_on(stream, x.device):
                    out = torch.empty((n, heads, shape.head_dim), dtype=dtype, device=x.device)
            _check_rows(out, name + "_out", n, heads, shape.head_dim, dtype, index)
        elif out is not None:
            raise ValueError(f"{name}_out without {name}")
        outs.append(out)
    with _on(index):
        aug_rope_rows(shape, rope.angles, positions, q, k, *outs, stream=stream)
    return tuple(outs)


class StepTables:
    """Tables of steps whose lengths are on the GPU: which blocks every request
    holds, and for the step's rows where they start, their positions, slots and (with
    ``max_draft``) the drafts of their request that each sees. All of them are device
    tensors that ``update`` writes in place, so that it can be captured in a graph
    together with what reads them. What stands behind the step's rows is of an earlier
    step: an append of ``max_rows`` rows takes ``live_rows`` (int32 [1]) along.

    ``max_reqs`` requests (unused ones have lengths 0), ``max_rows`` rows of one step,
    ``max_blocks`` columns of the table, a pool of ``num_pool_blocks``. Without
    ``block_table`` and ``held`` no request holds blocks; ``free_ids`` (int32
    [num_pool_blocks], the first ``free_count`` of which are free, all by default) stands
    for all blocks of the pool by default. Tensors given here are used, not copied."""

    def __init__(self, max_reqs: int, max_rows: int, max_blocks: int, num_pool_blocks: int, max_draft: int = MAX_DRAFT, device="cuda",
                 block_table: torch.Tensor = None, held: torch.Tensor = None, free_ids: torch.Tensor = None, free_count: int = None):
        device = torch.device(device)
        if (block_table is None) != (held is None) or (block_table is not None and free_ids is None):
            raise ValueError("a block table comes with what is held and which blocks are free")
        self.max_reqs, self.max_rows, self.max_blocks = int(max_reqs), int(max_rows), int(max_blocks)
        self.num_pool_blocks, self.max_draft = int(num_pool_blocks), int(max_draft)
        if free_count is None:
            free_count = self.num_pool_blocks
        if not 0 <= free_count <= self.num_pool_blocks:
            raise ValueError(f"{free_count} free blocks of {self.num_pool_blocks}")
        zeros = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        self.block_table = zeros(self.max_reqs, self.max_blocks) if block_table is None else block_table
        self.held = zeros(self.max_reqs) if held is None else held
        self.free_ids = torch.arange(self.num_pool_blocks, dtype=torch.int32, device=device) if free_ids is None else free_ids
        self.free_count = torch.full((1,), int(free_count), dtype=torch.int32, device=device)
        self.q_start, self.kv_len, self.state = zeros(self.max_reqs + 1), zeros(self.max_reqs), zeros(self.max_reqs)
        self.live_rows = self.q_start[self.max_reqs:]     # the step's rows
        self.positions, self.slots = zeros(self.max_rows), zeros(self.max_rows, dtype=torch.int64)
        self.seen = zeros(self.max_rows, dtype=torch.int64) if self.max_draft else None
        self._scratch = zeros(STEP_SCRATCH_BYTES, dtype=torch.uint8)
        self.device = self.q_start.device
        self._index = index = self.q_start.get_device()
        _check_vector(self.held, "held", self.max_reqs, torch.int32, index)
        _check_vector(self.free_ids, "free_ids", self.num_pool_blocks, torch.int32, index)
        t = self.block_table
        if t.shape != (self.max_reqs, self.max_blocks) or t.dtype != torch.int32 or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"block_table: contiguous int32 of shape ({self.max_reqs}, {self.max_blocks}) on {self.device}, got "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}")
        at = lambda x: None if x is None else x.data_ptr()  # noqa: E731
        self._args = aug_step_tables_args(
            self.max_reqs, self.max_rows, self.max_blocks, self.num_pool_blocks, self.max_draft, 0, None, None, None, at(t), at(self.held),
            at(self.free_ids), at(self.free_count), at(self.q_start), at(self.kv_len), at(self.state), at(self.positions),
            at(self.slots), at(self.seen), at(self._scratch))

    def update(self, ctx_len: torch.Tensor, q_len: torch.Tensor, parents: torch.Tensor = None, stream=None):
        """Enqueue the tables of a step of ``q_len`` rows a request after ``ctx_len``
        tokens in the cache (int32 [max_reqs]); ``parents`` (int32 [max_rows]): the row of
        the same request that each draft follows, -1 for a root; None: every row follows
        the one before. Blocks that requests no longer need are free again, new ones are
        taken. ``state`` says which requests were refused. ``ctx_len`` may be the tables' own
        ``kv_len`` (plain decoding: 0 for a request that was refused, whose blocks then come
        back); otherwise what is given here overlaps none of the tables."""
        index = self._index
        _check_vector(ctx_len, "ctx_len", self.max_reqs, torch.int32, index)
        _check_vector(q_len, "q_len", self.max_reqs, torch.int32, index)
        if parents is not None:
            _check_vector(parents, "parents", self.max_rows, torch.int32, index)
        a = self._args
        a.ctx_len, a.q_len = ctx_len.data_ptr(), q_len.data_ptr()
        a.parents = None if parents is None else parents.data_ptr()
        with _on(index):
            aug_step_tables(a, stream=_current_stream(index) if stream is None else stream)


_PLAN_HEADER_BYTES = 64


class TreeAttention:
    """Attention of a step's drafts over a paged cache, from ``StepTables``: ``plan``
    once a step, ``run`` once a layer. Its work list, workspace and output belong to it:
    layers that run at the same time need one each."""

    def __init__(self, shape, kv: PagedKV, tables: StepTables):
        if not tables.max_draft:
            raise ValueError("the tables keep no masks (max_draft 0)")
        if tables._index != kv._device or tables.num_pool_blocks != kv.num_pool_blocks:
            raise ValueError(f"tables of {tables.num_pool_blocks} blocks on {tables.device}, a pool of {kv.num_pool_blocks} on "
                             f"{kv.k_cache.device}")
        self.shape, self.kv, self.tables = shape, kv, tables
        self._index = kv._device
        self._check_pool(kv)
        self._planned = False
        t = tables
        self._batch = aug_tree_batch(t.max_reqs, t.max_rows, t.max_blocks, t.max_draft, t.q_start.data_ptr(), t.kv_len.data_ptr(),
                                     t.block_table.data_ptr(), t.seen.data_ptr())
        plan_bytes, workspace_bytes = aug_tree_plan_size(shape, self._batch)
        self.plan_dev = torch.empty(plan_bytes, dtype=torch.uint8, device=t.device)
        self.plan_dev[:_PLAN_HEADER_BYTES].zero_()       # an empty plan, where plan() has only been captured so far
        self.workspace = torch.empty(workspace_bytes, dtype=torch.uint8, device=t.device)
        self._rows = (t.max_rows, shape.num_q_heads, shape.head_dim)
        self._dtype = torch.float32 if shape.q_dtype == AUG_F32 else torch.bfloat16
        # zeros: rows behind the step's last are never written
        self.out = torch.zeros(self._rows, dtype=self._dtype, device=t.device)

    def plan(self, stream=None):
        """Enqueue the work list of the tables as they are then."""
        with _on(self._index):
            aug_tree_plan(self.shape, self._batch, self.plan_dev, stream=stream)
        self._planned = True

    def _check_pool(self, kv):
        for field in ("kv_dtype", "num_kv_heads", "head_dim"):
            if getattr(kv.shape, field) != getattr(self.shape, field):
                raise ValueError(f"a pool of {field} {getattr(kv.shape, field)}, the attention has {getattr(self.shape, field)}")

    def run(self, q: torch.Tensor, out: torch.Tensor = None, stream=None, kv: PagedKV = None):
        """Enqueue the attention of ``q`` ([max_rows][H_q][D], contiguous) into ``out``
        (the object's own by default; ``q`` itself will do), over ``kv`` (another layer's pool of the same
        size, or the planned one). Rows that see no key become zeros; rows behind the
        step's last are left as they were."""
        kv = self.kv if kv is None else kv
        out = self.out if out is None else out
        if kv.num_pool_blocks != self.kv.num_pool_blocks or kv._device != self._index:
            raise ValueError(f"a pool of {kv.num_pool_blocks} blocks, planned for {self.kv.num_pool_blocks}")
        if kv is not self.kv:
            self._check_pool(kv)
        if not self._planned:
            raise ValueError("no step has been planned")
        for name, t in (("q", q), ("out", out)):
            if t.shape != self._rows or t.dtype != self._dtype or not t.is_contiguous() or t.get_device() != self._index:
                raise ValueError(f"{name}: contiguous {self._dtype} of shape {self._rows} on {self.tables.device}, got {t.dtype} "
                                 f"{tuple(t.shape)} on {t.device}")
        with _on(self._index):
            aug_attn_tree(self.shape, self._batch, self.plan_dev, q, kv.k_cache, kv.v_cache, kv.k_scale, kv.v_scale,
                          kv.num_pool_blocks, out, self.workspace, stream=stream)
        return out


def sample(logits: torch.Tensor, uniform: torch.Tensor, temperature: torch.Tensor = None, top_k: torch.Tensor = None,
           top_p: torch.Tensor = None, min_p: torch.Tensor = None, tokens: torch.Tensor = None, probs: torch.Tensor = None, stream=None):
    """One token for each row of ``logits`` ([rows][vocab], float32 or bf16; rows may be
    strided) from ``uniform`` (float32 [rows] in [0, 1)), with a ``temperature`` (float32,
    0: greedy), ``top_k`` (int32, 0: all), ``top_p`` and ``min_p`` (float32) of each row, or None.
    Returns (tokens int32, probs float32: each token's share of what was kept), allocated
    on ``stream`` where they are not given. What exactly is drawn stands in aug.h."""
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or logits.get_device() < 0 or \
            (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits: float32 or bf16 rows of contiguous logits on a GPU, got {logits.dtype} {tuple(logits.shape)}, strides "
                         f"{logits.stride()} on {logits.device}")
    rows, vocab = logits.shape
    index = logits.get_device()
    _check_vector(uniform, "uniform", rows, torch.float32, index)
    for name, t, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                           ("min_p", min_p, torch.float32), ("tokens", tokens, torch.int32), ("probs", probs, torch.float32)):
        if t is not None:
            _check_vector(t, name, rows, dtype, index)
    if tokens is None or probs is None:
        with _allocating_on(stream, logits.device):
            tokens = torch.empty(rows, dtype=torch.int32, device=logits.device) if tokens is None else tokens
            probs = torch.empty(rows, dtype=torch.float32, device=logits.device) if probs is None else probs
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = aug_sample_args(rows, vocab, AUG_F32 if logits.dtype == torch.float32 else AUG_BF16, 0, max(logits.stride(0), vocab) if rows < 2 else
                           logits.stride(0), logits.data_ptr(), uniform.data_ptr(), at(temperature), at(top_k), at(top_p), at(min_p),
                           tokens.data_ptr(), probs.data_ptr())
    with _on(index):
        aug_sample(args, stream=_current_stream(index) if stream is None else stream)
    return tokens, probs


class MixedAttention:
    """One planned mixed batch: its plan image and workspace on the device,
    its output tensor, and the launch."""

    def __init__(self, shape, kv: PagedKV, q_start, ctx_len, bt_start, block_ids_host,
                 block_ids_dev: torch.Tensor, kv_split_tokens: int = 0, check_blocks: bool = True,
                 row_path: int = 0, tile_path: int = 0, row_first=None, row_end=None):
        """``row_first`` and ``row_end`` (host, one entry per query row): the
        keys that each row sees instead of the causal ones (``row_spans`` makes
        them)."""
        self.shape, self.kv = shape, kv
        device = kv.k_cache.device
        self.info, plan = aug_attn_plan(shape, q_start, ctx_len, bt_start, kv.num_pool_blocks,
                                        block_ids_host if check_blocks else None,
                                        kv_split_tokens=kv_split_tokens, row_path=row_path,
                                        tile_path=tile_path, row_first=row_first, row_end=row_end)
        # pinned staging kept alive with the batch; the library's copy kernel
        # moves it on the current stream of the cache's device
        self.plan_host = torch.from_numpy(plan.copy()).pin_memory()
        self.plan_dev = torch.empty(max(1, plan.size), dtype=torch.uint8, device=device)
        aug_plan_upload(self.plan_host, self.plan_dev, plan.size)
        self.workspace = torch.empty(max(256, int(self.info.workspace_bytes)), dtype=torch.uint8,
                                     device=device)
        self.block_ids = block_ids_dev
        rows = int(self.info.total_rows)
        out_dtype = torch.float32 if shape.out_dtype == 0 else torch.bfloat16
        self.out = torch.empty((rows, shape.num_q_heads, shape.head_dim), dtype=out_dtype, device=device)
        # what append() asks of the new K/V rows
        self._new_shape = (rows, shape.num_kv_heads, shape.head_dim)
        self._new_dtype = torch.float32 if shape.kv_dtype == 0 else torch.bfloat16

    def run(self, q: torch.Tensor, stream=None, kv: "PagedKV" = None, block_ids: torch.Tensor = None,
            out: torch.Tensor = None, softcap: float = 0.0, slopes: torch.Tensor = None):
        """Enqueue the batch's attention. ``kv``, ``block_ids`` and ``out``
        default to the planned ones; another layer of the same batch passes its
        own pool, block ids (same table shape) and output, and reuses the plan.
        ``softcap``: scores become softcap * tanh(score / softcap); ``slopes``
        (float32 [num_q_heads]): less slope * |position - key|. ``stream`` has to
        wait for the stream that was torch's current one when the batch was
        planned: its plan is uploaded and its memory allocated there."""
        kv = self.kv if kv is None else kv
        out = self.out if out is None else out
        if slopes is not None and (slopes.shape != (self.shape.num_q_heads,) or slopes.dtype != torch.float32 or
                                   slopes.device != q.device or not slopes.is_contiguous()):
            raise ValueError(f"slopes must be contiguous float32 of shape ({self.shape.num_q_heads},) on {q.device}, got "
                             f"{slopes.dtype} {tuple(slopes.shape)} on {slopes.device}")
        aug_attn_mixed(self.shape, self.info, self.plan_dev, q, kv.k_cache, kv.v_cache,
                       kv.k_scale, kv.v_scale, self.block_ids if block_ids is None else block_ids,
                       kv.num_pool_blocks, out, self.workspace, stream=stream, softcap=softcap, slopes=slopes)
        return out

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, stream=None, kv: "PagedKV" = None,
               block_ids: torch.Tensor = None):
        """Write the batch's new K/V rows ([rows][H_kv][D]) into the pool
        (``kv`` and ``block_ids`` as for ``run``)."""
        kv = self.kv if kv is None else kv
        want, dtype = self._new_shape, self._new_dtype
        for t in (k_new, v_new):
            if t.shape != want or t.dtype != dtype or not t.is_contiguous():
                raise ValueError(f"new K/V rows must be contiguous {dtype} of shape {want}, got "
                                 f"{t.dtype} {tuple(t.shape)}")
        aug_kv_append(self.shape, self.info, self.plan_dev, k_new, v_new, kv.k_cache,
                      kv.v_cache, kv.k_scale, kv.v_scale, self.block_ids if block_ids is None else block_ids,
                      kv.num_pool_blocks, stream=stream)


def row_spans(q_start, ctx_len, window: int = 0, prefix_len=None, doc_start=None):
    """(row_first, row_end) of a batch's query rows, which ``MixedAttention``
    takes: causal, and

    * ``window`` > 0: the row's own key and the window - 1 before it;
    * ``prefix_len`` (per request): keys before it are seen by every row of the
      request, later ones causally;
    * ``doc_start`` (per row): no key before it, the first of the row's document,
      nor of a prefix.

    A window and a prefix do not go together: a row behind both sees two spans.
    """
    if window > 0 and prefix_len is not None:
        raise ValueError("a window and a prefix: a row's keys are not one span")
    if window < 0:
        raise ValueError(f"a window of {window} keys (0: none)")
    q_start, ctx_len = np.asarray(q_start, np.int64), np.asarray(ctx_len, np.int64)
    q_len = np.diff(q_start)
    pos = np.arange(int(q_start[-1])) - np.repeat(q_start[:-1] - (ctx_len - q_len), q_len)
    first, end = np.zeros_like(pos), pos + 1
    if window > 0:
        first = np.maximum(first, end - window)
    if prefix_len is not None:
        end = np.maximum(end, np.repeat(np.minimum(prefix_len, ctx_len), q_len))
    if doc_start is not None:
        first = np.maximum(first, np.asarray(doc_start, np.int64))
    return first.astype(np.int32), end.astype(np.int32)


def shape_of(batch) -> object:
    return make_shape(batch.num_q_heads, batch.num_kv_heads, batch.head_dim, batch.q_dtype,
                      batch.kv_dtype, batch.out_dtype, batch.softmax_scale)


def upload_batch(batch, device="cuda", staging_bytes=1 << 28):
    """Move a host batch (fields as produced by the seeded generators) to the
    device: returns (shape, PagedKV, q tensor, block_ids tensor)."""
    shape = shape_of(batch)
    k = to_device_array(batch.k_cache, batch.kv_dtype, device)
    v = to_device_array(batch.v_cache, batch.kv_dtype, device)
    ks = vs = None
    if batch.kv_dtype == "fp8":
        ks = torch.from_numpy(batch.k_scale).to(device)
        vs = torch.from_numpy(batch.v_scale).to(device)
    kv = PagedKV(shape, k, v, ks, vs, staging_bytes=staging_bytes)
    q = to_device_array(batch.q, batch.q_dtype, device)
    bids = torch.from_numpy(np.ascontiguousarray(batch.block_ids, dtype=np.int32)).to(device)
    return shape, kv, q, bids


def serving_former(**params):
    """A batch former for the serving loop (``synth.trace.ServingLoop``):
    ``former(records, free_blocks, now)`` packs the records (dicts with the
    request-record field names) into the library's request layout, calls
    ``aug_form_batch`` and returns its plan dict. ``params`` are the fields of
    the former's parameter record."""
    from . import REQUEST_DTYPE, aug_form_batch, former_params
    p = former_params(**params)
    names = REQUEST_DTYPE.names

    def run(recs, free_blocks, now):
        arr = np.zeros(len(recs), REQUEST_DTYPE)
        for k in names:
            if k != "reserved":
                arr[k] = [r[k] for r in recs]
        t0 = time.perf_counter()
        plan = aug_form_batch(arr, free_blocks, now, p)
        run.timings.append((time.perf_counter() - t0, len(recs), int(np.count_nonzero(arr["state"] == 3))))
        return plan
    # (seconds in the library call, records, paused records) per iteration
    run.timings = []
    return run


class _LibraryLifecycle:
    """Request records of a serving loop, created and renewed by the library
    (Algorithm 1, steps (1)-(2)). Records are dicts with the field names of
    the library's request record."""

    def __init__(self):
        from . import REQUEST_DTYPE
        self.dtype = REQUEST_DTYPE
        self.names = [k for k in REQUEST_DTYPE.names if k != "reserved"]

    def _dict(self, rec):
        return {k: rec[k].item() for k in self.names}

    def arrive(self, id, arrival, prompt_tokens, pred_out, pred_call, has_next_call):
        from . import aug_request_arrive
        return self._dict(aug_request_arrive(id, arrival, prompt_tokens, pred_out, pred_call, has_next_call))

    def on_return(self, rec, realised, context_tokens, ret_tokens, pred_out, pred_call, has_next_call):
        from . import aug_request_return
        arr = np.zeros(1, self.dtype)
        for k in self.names:
            arr[0][k] = rec[k]
        return self._dict(aug_request_return(arr[0], realised, context_tokens, ret_tokens, pred_out,
                                             pred_call, has_next_call))


def serving_lifecycle():
    """The library's request-record transitions for ``synth.trace.ServingLoop``."""
    return _LibraryLifecycle()
