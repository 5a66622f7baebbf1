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

from . import (AUG_F32, AUG_MXFP4, MXFP4_CELL_BYTES, aug_attn_mixed, aug_attn_plan, aug_kv_append, aug_kv_park, aug_kv_read,
               aug_kv_record_bytes, aug_kv_resume, aug_plan_upload, make_shape)

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
