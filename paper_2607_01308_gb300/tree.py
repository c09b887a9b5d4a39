"""Torch-facing side of the operators around a tree of drafted tokens (cm_qcache_tree, cm_qk_rotate and
cm_tree_verify of include/cm.h): argument checks and marshalling only, in few interpreter steps, as in qcache.py."""
from __future__ import annotations

import struct
from typing import Optional, Tuple

from ._binding import CM_PROB_BF16, CM_PROB_F32, Context, _check, _stream_handle, lib
from .qcache import QBatch, _fixed, _new_on, _require, _strides

_pack_rows = struct.Struct("@PPPPPPPqqqqqqqqqiiifi4x").pack      # a cm_qk_rows in one step
_pack_drafts = struct.Struct("@PPPPPPPPPPqqiiiii4x").pack        # a cm_tree_drafts


class QTree:
    """Trees of drafted tokens, one for each request of a batch: what is known of their rows, on the GPU.

      mask [max_rows, words] int32 (bit j: row j of the request is the row or an ancestor) and positions [max_rows]
      int32: written by plan()
      path [max_rows], kept [R], next_token [R] int32: written by verify(), the accepted rows of each request, from
      its first row's place on, their number and the token behind them
      lens [R] int32, freed [max_freed] int32, freed_count [1] int64: written by QCache.keep(), the tokens that
      each request holds then, the blocks that none is left in (-1 behind the last) and their number

    max_nodes: the most rows of one request, to 256; rows behind it are seen by none and never accepted. max_freed: entries of
    freed, if not one for each request and one for each block_size rows of the batch. Those hold the blocks of any step whose rows
    all had room in the batch. schedule() takes blocks for the rows that max_rows cuts off too, which keep() gives back:
    a program whose steps may be cut asks for num_requests * table_width, which is always enough. freed_count counts
    what there was no room for as well; those blocks are still named by the table, behind what lens needs, until schedule()
    writes others over them. A program with masks or
    paths of its own writes into these tensors instead. One tree is used by one stream at a time; its memory is
    given back as a QBatch's is."""

    mask, positions, path, kept = _fixed("_mask"), _fixed("_positions"), _fixed("_path"), _fixed("_kept")
    next_token, lens = _fixed("_next_token"), _fixed("_lens")
    freed, freed_count = _fixed("_freed"), _fixed("_freed_count")

    def __init__(self, batch: QBatch, max_nodes: int, max_freed: Optional[int] = None):
        import torch
        _require(1 <= max_nodes <= 256, "max_nodes must be in [1, 256]")
        _require(max_freed is None or 0 <= max_freed < 1 << 31, "max_freed must be in [0, 2^31 - 1]")
        dev = batch.row_starts.device
        rows, n = batch.slot_map.numel(), batch._num_requests
        self.batch, self.ctx = batch, batch.ctx
        self.max_nodes = max_nodes
        self._device, self._max_rows, self._num_requests = batch._device, rows, n
        self._words, self._max_freed = (max_nodes + 31) // 32, n + rows // batch._c.block_size if max_freed is None else max_freed
        self._int32, self._fp32, self._bf16 = torch.int32, torch.float32, torch.bfloat16

        def whole(*shape, fill=-1, dtype=torch.int32):
            return torch.full(shape, fill, dtype=dtype, device=dev)

        self._mask, self._positions = whole(rows, self._words, fill=0), whole(rows, fill=0)
        self._path, self._kept, self._next_token = whole(rows), whole(n, fill=0), whole(n)
        self._lens, self._freed, self._freed_count = whole(n, fill=0), whole(self._max_freed), whole(1, fill=0, dtype=torch.int64)
        self._mask_ptr, self._positions_ptr = self._mask.data_ptr() or None, self._positions.data_ptr() or None
        self._path_ptr, self._kept_ptr, self._next_ptr = self._path.data_ptr() or None, self._kept.data_ptr() or None, self._next_token.data_ptr() or None
        self._lens_ptr, self._freed_ptr, self._count_ptr = self._lens.data_ptr() or None, self._freed.data_ptr() or None, self._freed_count.data_ptr()
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(dev).synchronize()      # set on every stream
        self._streams = {_stream_handle(torch.cuda.current_stream(dev))}

    def _on(self, stream) -> Optional[int]:
        """The stream's handle; the first time, its use of the tree's memory is made known to torch."""
        handle = _stream_handle(stream)
        if handle not in self._streams and not isinstance(stream, int):
            import torch
            stream = stream or torch.cuda.current_stream(self._device)
            for t in (self._mask, self._positions, self._path, self._kept, self._next_token, self._lens, self._freed, self._freed_count):
                t.record_stream(stream)
            self._streams.add(handle)
        return handle

    def _vector(self, t, dtype, n, what: str):
        if t.dtype is not dtype or t.dim() != 1 or not t.is_contiguous() or t.numel() != n or t.get_device() != self._device:
            raise ValueError(what)
        return t.data_ptr() or None

    def plan(self, parents, context_lens, stream=None) -> "QTree":
        """mask and positions from the rows' parents (int32 CUDA tensor [rows], at most as many as the batch has; the
        place of each row's parent among its request's rows, -1 for none) and the tokens in front of each request's rows
        (int32 [R]). parents None: every row follows the one before it."""
        rows = self._max_rows
        if parents is not None:
            rows = parents.numel()
            _require(rows <= self._max_rows, "more parents than the batch has rows")
            parents = self._vector(parents, self._int32, rows, "parents must be a contiguous int32 vector on the context's device")
        context = self._vector(context_lens, self._int32, self._num_requests,
                               "context_lens must be a contiguous int32 vector with a length for each request, on the context's device")
        self.batch._on(stream)
        _check(lib.cm_qcache_tree(self.ctx.handle, self.batch._ref, context, parents, rows, self._words, self._mask_ptr,
                                  self._positions_ptr, self._on(stream)))
        return self

    def verify(self, parents, tokens, target, accept, sample, draft=None, stream=None) -> "QTree":
        """path, kept and next_token from the drafted tokens (int32 [rows]), the target's probabilities of what follows each row,
        those that the rows behind it were drawn from (target, draft: fp32 or bf16 [rows, vocab], vocab contiguous; draft
        None: drafted without chance) and uniform random numbers of [0, 1): accept [rows], sample [R] (fp32). What is
        accepted and chosen is distributed as the target's own tokens are."""
        rows, shape, dtype, device = parents.numel(), target.shape, target.dtype, self._device
        _require(rows <= self._max_rows, "more parents than the batch has rows")
        if (dtype is not self._fp32 and dtype is not self._bf16) or len(shape) != 2 or shape[0] < rows or target.get_device() != device:
            raise ValueError("target must be fp32 or bf16 [rows, vocab] on the context's device")
        if draft is not None and (draft.dtype is not dtype or draft.shape != shape or draft.get_device() != device):
            raise ValueError("draft must be like target")
        if shape[1] > 1 and (target.stride(1) != 1 or (draft is not None and draft.stride(1) != 1)):
            raise ValueError("the vocabulary must be contiguous")
        what = "parents and tokens (int32), accept (fp32) must be contiguous vectors of the same size, sample (fp32) one with a number for each request, on the context's device"
        int32, fp32 = self._int32, self._fp32
        parents, tokens = self._vector(parents, int32, rows, what), self._vector(tokens, int32, rows, what)
        accept, sample = self._vector(accept, fp32, rows, what), self._vector(sample, fp32, self._num_requests, what)
        batch = self.batch
        drafts = _pack_drafts(batch._c.row_starts, parents or 0, tokens or 0, target.data_ptr(), 0 if draft is None else draft.data_ptr(), accept or 0,
                              sample or 0, self._path_ptr or 0, self._kept_ptr or 0, self._next_ptr or 0, target.stride(0),
                              0 if draft is None else draft.stride(0), self._num_requests, rows, shape[1], self.max_nodes,
                              CM_PROB_F32 if dtype is fp32 else CM_PROB_BF16)
        batch._on(stream)
        _check(lib.cm_tree_verify(self.ctx.handle, drafts, self._on(stream)))
        return self


_ROWS = "q and k must be bf16 [rows, heads, head_dim] of the same rows and head_dim, contiguous in it, on the context's device"


def _weight(t, bf16, d: int, device: int) -> int:
    if t.dtype is not bf16 or t.dim() != 1 or t.numel() != d or not t.is_contiguous() or t.get_device() != device:
        raise ValueError("weights must be contiguous bf16 [head_dim] on the context's device")
    return t.data_ptr()


def rotate_qk(ctx: Context, q, k, positions, q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None, k_out=None,
              stream=None) -> Tuple[object, object]:
    """(q_out, k_out): every head's row of q and k (bf16 CUDA tensors [rows, heads, head_dim], head_dim contiguous; views of a
    fused projection, say), normed (x / sqrt(mean x^2 + eps) * weight; a weight of None: not) and rotated to
    positions [rows] (int32) by the angles of a fragment's keys, with the context's rope_theta, in fp32. Either of q and k may be None. q_out
    and k_out are made if not given, on `stream`; they may be q and k themselves."""
    import torch
    _require(q is not None or k is not None, "q or k must be given")
    bf16, device, shape = torch.bfloat16, ctx.device, (k if q is None else q).shape
    rows, d = shape[0], shape[-1]
    if (positions.dtype is not torch.int32 or positions.dim() != 1 or not positions.is_contiguous() or positions.numel() != rows or
            positions.get_device() != device):
        raise ValueError("positions must be a contiguous int32 vector with one for each row, on the context's device")
    q_in = q_to = qw = q_row = q_head = q_to_row = q_to_head = q_heads = 0
    k_in = k_to = kw = k_row = k_head = k_to_row = k_to_head = k_heads = 0
    if q is not None:
        if q.dtype is not bf16 or len(shape) != 3 or q.stride(2) != 1 or q.get_device() != device:
            raise ValueError(_ROWS)
        if q_out is None:
            q_out = _new_on(stream, q)
        elif q_out.dtype is not bf16 or q_out.shape != shape or q_out.stride(2) != 1 or q_out.get_device() != device:
            raise ValueError("q_out must be like q")
        if q_weight is not None:
            qw = _weight(q_weight, bf16, d, device)
        q_in, q_to, q_heads = q.data_ptr(), q_out.data_ptr(), shape[1]
        (q_row, q_head), (q_to_row, q_to_head) = _strides(q, 2, 8), _strides(q_out, 2, 8)
    else:
        _require(q_out is None and q_weight is None, "q_out or q_weight without q")
    if k is not None:
        shape = k.shape
        if k.dtype is not bf16 or len(shape) != 3 or shape[0] != rows or shape[2] != d or k.stride(2) != 1 or k.get_device() != device:
            raise ValueError(_ROWS)
        if k_out is None:
            k_out = _new_on(stream, k)
        elif k_out.dtype is not bf16 or k_out.shape != shape or k_out.stride(2) != 1 or k_out.get_device() != device:
            raise ValueError("k_out must be like k")
        if k_weight is not None:
            kw = _weight(k_weight, bf16, d, device)
        k_in, k_to, k_heads = k.data_ptr(), k_out.data_ptr(), shape[1]
        (k_row, k_head), (k_to_row, k_to_head) = _strides(k, 2, 8), _strides(k_out, 2, 8)
    else:
        _require(k_out is None and k_weight is None, "k_out or k_weight without k")
    _check(lib.cm_qk_rotate(ctx.handle, _pack_rows(q_in, k_in, q_to, k_to, qw, kw, positions.data_ptr(), q_row, q_head, k_row, k_head, q_to_row,
                                                   q_to_head, k_to_row, k_to_head, rows, q_heads, k_heads, d, eps, 0), _stream_handle(stream)))
    return q_out, k_out
