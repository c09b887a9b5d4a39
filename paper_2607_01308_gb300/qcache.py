"""Torch-facing side of the 8-bit paged cache (cm_qcache_* of include/cm.h): argument checks and
marshalling only. torch holds the memory; the library reads and writes it in place.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from ._binding import (Context, _check, _stream_handle, cm_qcache, cm_qcache_append, cm_qcache_batch,
                       cm_qcache_query, cm_qcache_schedule, cm_qcache_workspace, lib)

_INT8, _E4M3 = 1, 0


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _device(ctx: Context):
    import torch
    return torch.device("cuda", ctx.device)


def _strides(t, n: int, unit: int):
    """The first n strides of t; where a dimension has one entry its stride means nothing, and a
    multiple of `unit` stands for it."""
    return [s if t.shape[i] > 1 else t.shape[-1] * unit for i, s in enumerate(t.stride()[:n])]


def _same_layout(a, b, n: int) -> bool:
    return a.shape == b.shape and _strides(a, n, 1) == _strides(b, n, 1)


def _on_device(ctx: Context, t, what: str) -> None:
    _require(t.is_cuda and t.device.index == ctx.device, f"{what} must be on the context's device")


def _format(dtype) -> int:
    import torch
    _require(dtype in (torch.float8_e4m3fn, torch.int8), "a cache holds float8_e4m3fn or int8 codes")
    return _INT8 if dtype == torch.int8 else _E4M3


class QBatch:
    """The requests of a step: block table, row starts and lengths on the GPU, the slots of the new
    rows and the attention's workspace. One batch is used by one stream at a time.

      block_table [R, table_width] int32, row_starts [R + 1] int32, kv_lens [R] int32,
      slot_map [max_rows] int64, counts [2] int64 (blocks needed, rows)

    schedule() fills them; a program with tables of its own writes into them instead. max_new (host):
    the most new rows of one request that are expected (None: max_rows); attend() chooses its
    kernel by it, results do not depend on it."""

    def __init__(self, ctx: Context, num_requests: int, table_width: int, max_rows: int,
                 block_size: int):
        import torch
        _require(num_requests >= 0 and table_width >= 0 and max_rows >= 0, "sizes must not be negative")
        dev = _device(ctx)
        self.ctx = ctx
        self.max_rows = max_rows
        self.max_new: Optional[int] = None
        self.block_table = torch.full((num_requests, table_width), -1, dtype=torch.int32, device=dev)
        self.row_starts = torch.zeros(num_requests + 1, dtype=torch.int32, device=dev)
        self.kv_lens = torch.zeros(num_requests, dtype=torch.int32, device=dev)
        self.slot_map = torch.full((max_rows,), -1, dtype=torch.int64, device=dev)
        self.counts = torch.zeros(2, dtype=torch.int64, device=dev)
        self._c = cm_qcache_batch(num_requests, block_size, table_width, self.block_table.data_ptr() or None,
                                  self.row_starts.data_ptr(), self.kv_lens.data_ptr() or None)
        self._ref = ctypes.byref(self._c)
        self._workspace = None
        self._workspace_dim = 0

    def schedule(self, context_lens, new_lens, free_blocks, stream=None) -> "QBatch":
        """Block tables, row starts, lengths and slots from the requests' cached and new token counts
        (int32 CUDA tensors [R]); new blocks come from the front of free_blocks (int32)."""
        import torch
        for t, what in ((context_lens, "context_lens"), (new_lens, "new_lens"), (free_blocks, "free_blocks")):
            _require(t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous(), f"{what} must be a contiguous int32 vector")
            _on_device(self.ctx, t, what)
        n = self._c.num_requests
        _require(len(context_lens) == n and len(new_lens) == n, "one length per request")
        cm_qcache_schedule(self.ctx.handle, self._c, context_lens.data_ptr() or None, new_lens.data_ptr() or None,
                           free_blocks.data_ptr() or None, len(free_blocks), self.slot_map.data_ptr() or None,
                           self.max_rows, self.counts.data_ptr(), stream)
        return self

    def _space(self, head_dim: int):
        import torch
        need = cm_qcache_workspace(self.ctx.handle, head_dim)
        self._workspace = torch.zeros(need, dtype=torch.uint8, device=_device(self.ctx))
        torch.cuda.current_stream(self._workspace.device).synchronize()   # zero on every stream
        self._workspace_dim = head_dim
        return self._workspace


class QCache:
    """A paged KV cache held in 8 bits: codes k, v [num_blocks, layers, kv_heads, block_size, head_dim]
    (float8_e4m3fn or int8) and one fp32 scale for each block, layer and head, k_scale, v_scale
    [num_blocks, layers, kv_heads]; a stored value is code * scale."""

    def __init__(self, ctx: Context, num_blocks: int, block_size: int, num_layers: int,
                 num_kv_heads: int, head_dim: int, dtype=None):
        import torch
        dtype = dtype or torch.float8_e4m3fn
        _format(dtype)
        dev = _device(ctx)
        shape = (num_blocks, num_layers, num_kv_heads, block_size, head_dim)
        self._set(ctx, torch.zeros(shape, dtype=torch.uint8, device=dev).view(dtype),
                  torch.zeros(shape, dtype=torch.uint8, device=dev).view(dtype),
                  torch.zeros(shape[:3], device=dev), torch.zeros(shape[:3], device=dev))

    @classmethod
    def from_tensors(cls, ctx: Context, k, v, k_scale, v_scale) -> "QCache":
        """A cache in the caller's own tensors, of any strides with head_dim contiguous (a permuted
        view of another layout, say); k and v alike, k_scale and v_scale alike."""
        self = cls.__new__(cls)
        self._set(ctx, k, v, k_scale, v_scale)
        return self

    def _set(self, ctx, k, v, k_scale, v_scale):
        import torch
        fmt = _format(k.dtype)
        _require(k.dim() == 5 and k.shape == v.shape and k.dtype == v.dtype, "k and v must both be [blocks, layers, kv_heads, block_size, head_dim]")
        _require(_same_layout(k, v, 4) and k.stride(4) == 1, "k and v must have the same strides, head_dim contiguous")
        _require(k_scale.dtype == torch.float32 and v_scale.dtype == torch.float32 and
                 tuple(k_scale.shape) == tuple(k.shape[:3]) and tuple(v_scale.shape) == tuple(k.shape[:3]) and
                 _same_layout(k_scale, v_scale, 3), "scales must be fp32 [blocks, layers, kv_heads] of the same strides")
        for t in (k, v, k_scale, v_scale):
            _on_device(ctx, t, "cache tensors")
        self.ctx, self.k, self.v, self.k_scale, self.v_scale = ctx, k, v, k_scale, v_scale
        nb, L, H, bs, d = k.shape
        s, z = _strides(k, 4, 16), _strides(k_scale, 3, 1)
        self._c = cm_qcache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), fmt, L, H, d, bs, 0,
                            nb, s[0], s[1], s[2], s[3], z[0], z[1], z[2])
        self._query = cm_qcache_query()
        self._query_ref = ctypes.byref(self._query)
        self._ref = ctypes.byref(self._c)

    def append(self, K, V, slot_map, layer: int = 0, stream=None) -> None:
        """Rows K, V (bf16 CUDA tensors [layers, kv_heads, rows, head_dim] of the same strides, head_dim
        contiguous) into the slots [rows] (int64) of layers layer .. layer + layers - 1. A slot of -1 is
        skipped; slots of one block are consecutive and ascending."""
        import torch
        n = slot_map.shape[0]
        _require(K.dtype == torch.bfloat16 and V.dtype == torch.bfloat16 and K.dim() == 4 and K.shape == V.shape and
                 K.shape[1] == self._c.num_kv_heads and K.shape[3] == self._c.head_dim,
                 "K and V must be bf16 [layers, kv_heads, rows, head_dim] of the cache's shape")
        _require(_same_layout(K, V, 3) and K.stride(3) == 1, "K and V must have the same strides, head_dim contiguous")
        _require(slot_map.dtype == torch.int64 and slot_map.dim() == 1 and slot_map.is_contiguous() and n <= K.shape[2],
                 "slot_map must be a contiguous int64 vector of at most as many entries as there are rows")
        for t in (K, V, slot_map):
            _on_device(self.ctx, t, "rows and slots")
        s = _strides(K, 3, 8)
        cm_qcache_append(self.ctx.handle, self._c, layer, K.shape[0], K.data_ptr() or None, V.data_ptr() or None,
                         s[0], s[1], s[2], slot_map.data_ptr() or None, n, stream)

    def attend(self, q, batch: QBatch, layer: int = 0, out=None, lse=None, softmax_scale: Optional[float] = None,
               causal: bool = True, stream=None) -> Tuple[object, object]:
        """(out, lse): softmax(softmax_scale * q K^T) V for the batch's rows, each over its own request's
        cached tokens. q, out: bf16 [rows, q_heads, head_dim] (q_heads a multiple of kv_heads, head_dim
        contiguous); lse: fp32 [rows, q_heads] or None to leave it out; out is made if not given."""
        import torch
        shape = q.shape
        _require(q.dtype == torch.bfloat16 and q.dim() == 3 and shape[2] == self._c.head_dim and q.stride(2) == 1,
                 "q must be bf16 [rows, q_heads, head_dim], head_dim contiguous")
        _on_device(self.ctx, q, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        else:
            _require(out.dtype == torch.bfloat16 and out.shape == shape and out.stride(2) == 1 and out.device == q.device,
                     "out must be like q")
        if lse is not None:
            _require(lse.dtype == torch.float32 and lse.shape == shape[:2] and lse.is_contiguous() and lse.device == q.device,
                     "lse must be a contiguous fp32 [rows, q_heads]")
        space = batch._workspace
        if space is None or batch._workspace_dim < self._c.head_dim:
            space = batch._space(self._c.head_dim)
        c, qs, os = self._query, _strides(q, 2, 8), _strides(out, 2, 8)
        c.q, c.out, c.lse = q.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else None
        c.q_stride_row, c.q_stride_head, c.out_stride_row, c.out_stride_head = qs[0], qs[1], os[0], os[1]
        c.total_rows, c.num_q_heads = shape[0], shape[1]
        c.max_rows_per_request = batch.max_new or 0
        c.causal = 1 if causal else 0
        c.softmax_scale = softmax_scale if softmax_scale is not None else self._c.head_dim ** -0.5
        _check(lib.cm_qcache_attend(self.ctx.handle, self._ref, layer, batch._ref, self._query_ref,
                                    space.data_ptr(), space.numel(), _stream_handle(stream)))
        return out, lse
