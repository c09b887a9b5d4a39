"""Torch-facing side of the 8-bit paged cache (cm_qcache_* of include/cm.h): argument checks and
marshalling only. torch holds the memory; the library reads and writes it in place.

A serving step makes these calls once for each layer, on kernels of a few microseconds: the
checks are written for few interpreter steps (messages are only built for a refusal, descriptors
of tensors that an object owns are filled once).
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

from ._binding import (CM_QCACHE_CONTEXT_LENS, Context, _check, _stream_handle, cm_qcache, cm_qcache_batch, cm_qcache_workspace,
                       lib)

_INT8, _E4M3 = 1, 0
_ATTENTION_DIMS = (32, 64, 128, 256)
_pack_query = struct.Struct("@PPPqqqqiiiifiP").pack    # a cm_qcache_query in one step


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _device(ctx: Context):
    import torch
    return torch.device("cuda", ctx.device)


def _strides(t, n: int, unit: int):
    """The first n strides of t; where a dimension has one entry its stride means nothing, and a
    multiple of `unit` stands for it."""
    shape, stride = t.shape, t.stride()[:n]
    if 1 not in shape:
        return stride
    return tuple([s if shape[i] > 1 else shape[-1] * unit for i, s in enumerate(stride)])


def _same_layout(a, b, n: int) -> bool:
    return a.shape == b.shape and (a.stride() == b.stride() or _strides(a, n, 1) == _strides(b, n, 1))


def _new_on(stream, q):
    """An empty tensor like q (its strides left aside) from the memory of the stream that will write it: what other
    streams may still do with that memory is done."""
    if stream is None:
        return q.new_empty(q.shape)
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, q.device) if stream else torch.cuda.default_stream(q.device)
    with torch.cuda.stream(stream):
        return q.new_empty(q.shape)


def _format(dtype) -> int:
    import torch
    _require(dtype in (torch.float8_e4m3fn, torch.int8), "a cache holds float8_e4m3fn or int8 codes")
    return _INT8 if dtype == torch.int8 else _E4M3


def _fixed(name: str):
    """A tensor whose address the library holds: it can be written into (+= too), but not replaced."""
    def keep(self, value):
        if value is not getattr(self, name):
            raise AttributeError("%s is the memory that the calls use: write into it" % name[1:])
    return property(lambda self: getattr(self, name), keep)


class QBatch:
    """The requests of a step: block table, row starts and lengths on the GPU, the slots of the new
    rows and the attention's workspace. One batch is used by one stream at a time.

      block_table [R, table_width] int32, row_starts [R + 1] int32, kv_lens [R] int32,
      slot_map [max_rows] int64, counts [2] int64 (blocks needed, rows),
      context_lens [R] int32: the tokens before the rows of a request that schedule() had to cut short (its
      table row or max_rows ended), else -1

    schedule() fills them; a program with tables of its own writes into them instead (and leaves
    context_lens at -1 where a request's rows are the last of its kv_lens tokens). max_new (host, not
    set by schedule()): the most new rows of one request that are expected; attend() chooses the kernel of the whole
    call by it, and is right whatever it says. None counts as all rows of the call: a step of single tokens
    then goes to the kernel for prompts, at some twice its time.

    The workspace (some 40 MB) is made with the batch and stays where it is, for every head_dim, so that
    graphs which were captured with the batch can be replayed as long as it lives. The batch's memory is
    given back when the torch streams that its calls ran on are through with it; a stream given as a bare handle has to be
    through with it before the batch is dropped."""

    block_table, row_starts, kv_lens = _fixed("_block_table"), _fixed("_row_starts"), _fixed("_kv_lens")
    context_lens, slot_map, counts = _fixed("_context_lens"), _fixed("_slot_map"), _fixed("_counts")

    @property
    def max_rows(self) -> int:
        return self._max_rows

    @max_rows.setter
    def max_rows(self, rows: int) -> None:
        _require(0 <= rows <= self._slot_map.numel(), "max_rows must not pass the slot map's size")
        self._max_rows = rows

    def __init__(self, ctx: Context, num_requests: int, table_width: int, max_rows: int,
                 block_size: int):
        import torch
        _require(num_requests >= 0 and table_width >= 0 and max_rows >= 0, "sizes must not be negative")
        dev = _device(ctx)
        self.ctx = ctx
        self._device, self._int32 = ctx.device, torch.int32
        self._max_rows = max_rows
        self.max_new: Optional[int] = None
        self._block_table = torch.full((num_requests, table_width), -1, dtype=torch.int32, device=dev)
        self._row_starts = torch.zeros(num_requests + 1, dtype=torch.int32, device=dev)
        self._kv_lens = torch.zeros(num_requests, dtype=torch.int32, device=dev)
        self._context_lens = torch.full((num_requests,), -1, dtype=torch.int32, device=dev)
        self._slot_map = torch.full((max_rows,), -1, dtype=torch.int64, device=dev)
        self._counts = torch.zeros(2, dtype=torch.int64, device=dev)
        self._c = cm_qcache_batch(num_requests, block_size, table_width, self.block_table.data_ptr() or None,
                                  self.row_starts.data_ptr(), self.kv_lens.data_ptr() or None)
        self._ref = ctypes.byref(self._c)
        self._num_requests, self._slots, self._count_ptr = num_requests, self.slot_map.data_ptr() or None, self.counts.data_ptr()
        self._context = self.context_lens.data_ptr()
        self._workspace_bytes = max(cm_qcache_workspace(ctx.handle, d) for d in _ATTENTION_DIMS)
        self._workspace = torch.zeros(self._workspace_bytes, dtype=torch.uint8, device=dev)
        self._workspace_ptr = self._workspace.data_ptr()
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(dev).synchronize()      # set on every stream
        self._streams = {_stream_handle(torch.cuda.current_stream(dev))}

    def _on(self, stream) -> Optional[int]:
        """The stream's handle; the first time, its use of the batch's memory is made known to torch."""
        handle = _stream_handle(stream)
        if handle not in self._streams and not isinstance(stream, int):
            import torch
            stream = stream or torch.cuda.current_stream(self._device)
            for t in (self.block_table, self.row_starts, self.kv_lens, self.context_lens, self.slot_map, self.counts,
                      self._workspace):
                t.record_stream(stream)
            self._streams.add(handle)
        return handle

    def schedule(self, context_lens, new_lens, free_blocks, stream=None) -> "QBatch":
        """Block tables, row starts, lengths and slots from the requests' cached and new token counts
        (int32 CUDA tensors [R]); new blocks come from the front of free_blocks (int32)."""
        n, dtype, device = self._num_requests, self._int32, self._device
        for t in (context_lens, new_lens, free_blocks):
            if t.dtype is not dtype or t.dim() != 1 or not t.is_contiguous() or t.get_device() != device:
                raise ValueError("context_lens, new_lens and free_blocks must be contiguous int32 vectors on the context's device")
        _require(context_lens.numel() == n and new_lens.numel() == n, "one length per request")
        _check(lib.cm_qcache_schedule_cut(self.ctx.handle, self._ref, context_lens.data_ptr() or None, new_lens.data_ptr() or None,
                                          free_blocks.data_ptr() or None, free_blocks.numel(), self._slots, self._max_rows,
                                          self._count_ptr, self._context or None, self._on(stream)))
        return self


class QCache:
    """A paged KV cache held in 8 bits: codes k, v [num_blocks, layers, kv_heads, block_size, head_dim]
    (float8_e4m3fn or int8) and one fp32 scale for each block, layer and head, k_scale, v_scale
    [num_blocks, layers, kv_heads]; a stored value is code * scale."""

    k, v, k_scale, v_scale = _fixed("_k"), _fixed("_v"), _fixed("_k_scale"), _fixed("_v_scale")

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
        _require(_same_layout(k, v, 5) and k.stride(4) == 1, "k and v must have the same strides, head_dim contiguous")
        _require(k_scale.dtype == torch.float32 and v_scale.dtype == torch.float32 and
                 tuple(k_scale.shape) == tuple(k.shape[:3]) and tuple(v_scale.shape) == tuple(k.shape[:3]) and
                 _same_layout(k_scale, v_scale, 3), "scales must be fp32 [blocks, layers, kv_heads] of the same strides")
        _require(all(t.is_cuda and t.get_device() == ctx.device for t in (k, v, k_scale, v_scale)),
                 "cache tensors must be on the context's device")
        self._device = ctx.device
        self._bf16, self._fp32, self._int64 = torch.bfloat16, torch.float32, torch.int64
        self.ctx, self._k, self._v, self._k_scale, self._v_scale = ctx, k, v, k_scale, v_scale
        nb, L, H, bs, d = k.shape
        s, z = _strides(k, 4, 16), _strides(k_scale, 3, 1)
        self._c = cm_qcache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), fmt, L, H, d, bs, 0,
                            nb, s[0], s[1], s[2], s[3], z[0], z[1], z[2])
        self._heads, self._dim, self._scale = H, d, d ** -0.5
        self._ref = ctypes.byref(self._c)

    def append(self, K, V, slot_map, layer: int = 0, stream=None) -> None:
        """Rows K, V (bf16 CUDA tensors [layers, kv_heads, rows, head_dim] of the same strides, head_dim
        contiguous) into the slots [rows] (int64) of layers layer .. layer + layers - 1. A slot of -1 is
        skipped; slots of one block are consecutive and ascending."""
        shape, bf16, device = K.shape, self._bf16, self._device
        if (K.dtype is not bf16 or V.dtype is not bf16 or len(shape) != 4 or shape != V.shape or
                shape[1] != self._heads or shape[3] != self._dim):
            raise ValueError("K and V must be bf16 [layers, kv_heads, rows, head_dim] of the cache's shape")
        s = K.stride()
        if s[3] != 1 or (s != V.stride() and not _same_layout(K, V, 4)):
            raise ValueError("K and V must have the same strides, head_dim contiguous")
        if slot_map.dtype is not self._int64 or slot_map.dim() != 1 or not slot_map.is_contiguous() or slot_map.numel() > shape[2]:
            raise ValueError("slot_map must be a contiguous int64 vector of at most as many entries as there are rows")
        if K.get_device() != device or V.get_device() != device or slot_map.get_device() != device:
            raise ValueError("rows and slots must be on the context's device")
        if 1 in shape:
            s = _strides(K, 3, 8)
        _check(lib.cm_qcache_append(self.ctx.handle, self._ref, layer, shape[0], K.data_ptr() or None, V.data_ptr() or None,
                                    s[0], s[1], s[2], slot_map.data_ptr() or None, slot_map.numel(), _stream_handle(stream)))

    def attend(self, q, batch: QBatch, layer: int = 0, out=None, lse=None, softmax_scale: Optional[float] = None,
               causal: bool = True, stream=None, tree=None) -> Tuple[object, object]:
        """(out, lse): softmax(softmax_scale * q K^T) V for the batch's rows, each over its own request's
        cached tokens. q, out: bf16 [rows, q_heads, head_dim] (q_heads a multiple of kv_heads, head_dim
        contiguous); lse: fp32 [rows, q_heads] or None to leave it out; out is made if not given, on `stream`.
        With a tree (QTree) a row sees the tokens in front of its request's rows and the rows in its mask, whatever
        `causal` says."""
        shape, bf16, device = q.shape, self._bf16, self._device
        if q.dtype is not bf16 or len(shape) != 3 or shape[2] != self._dim or q.stride(2) != 1 or q.get_device() != device:
            raise ValueError("q must be bf16 [rows, q_heads, head_dim] on the context's device, head_dim contiguous")
        if out is None:
            out = _new_on(stream, q)
        elif out.dtype is not bf16 or out.shape != shape or out.stride(2) != 1 or out.get_device() != device:
            raise ValueError("out must be like q")
        if lse is not None and (lse.dtype is not self._fp32 or lse.shape != shape[:2] or not lse.is_contiguous() or
                                lse.get_device() != device):
            raise ValueError("lse must be a contiguous fp32 [rows, q_heads]")
        if batch._device != device:
            raise ValueError("the batch must be on the cache's device")
        qs, os = _strides(q, 2, 8), _strides(out, 2, 8)
        query = _pack_query(q.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr(), qs[0], qs[1], os[0], os[1],
                            shape[0], shape[1], batch.max_new or 0, 1 if causal else 0,
                            self._scale if softmax_scale is None else softmax_scale, CM_QCACHE_CONTEXT_LENS, batch._context)
        if tree is None:
            _check(lib.cm_qcache_attend(self.ctx.handle, self._ref, layer, batch._ref, query,
                                        batch._workspace_ptr, batch._workspace_bytes, batch._on(stream)))
            return out, lse
        if tree._device != device or tree._max_rows < shape[0]:
            raise ValueError("the tree must be on the cache's device and have a mask for every row")
        tree._on(stream)
        _check(lib.cm_qcache_attend_tree(self.ctx.handle, self._ref, layer, batch._ref, query, tree._mask_ptr, tree._words,
                                         batch._workspace_ptr, batch._workspace_bytes, batch._on(stream)))
        return out, lse

    def keep(self, batch: QBatch, tree, context_lens, stream=None) -> None:
        """The rows that tree.path and tree.kept name to the front of their requests' rows, in every layer; tree.lens,
        tree.freed and tree.freed_count are written: the tokens that each request holds now, the blocks that none is left in, and
        their number. context_lens: as schedule() took them (int32 CUDA tensor [R], not tree.lens itself)."""
        n, device = batch._num_requests, self._device
        if (context_lens.dtype is not batch._int32 or context_lens.dim() != 1 or not context_lens.is_contiguous() or
                context_lens.numel() != n or context_lens.get_device() != device):
            raise ValueError("context_lens must be a contiguous int32 vector with a length for each request, on the context's device")
        if batch._device != device or tree._device != device or tree._num_requests != n:
            raise ValueError("batch and tree must be on the cache's device and have the same requests")
        tree._on(stream)
        _check(lib.cm_qcache_keep(self.ctx.handle, self._ref, batch._ref, context_lens.data_ptr() or None, tree._path_ptr,
                                  tree._kept_ptr, tree._max_rows, tree._lens_ptr, tree._freed_ptr, tree._max_freed,
                                  tree._count_ptr, batch._on(stream)))
