"""Python face of the 8-bit paged key/value cache (ks_kv8_* of
include/knapspec.h): torch allocates the memory, this module checks the
tensors and marshals their addresses and strides; the work runs in the
library's CUDA kernels.

    cache = Cache8(n_pages, page_tokens, n_kv_heads, head_dim)
    batch = Batch8(page_table, row_offsets, lengths, n_rows)
    cache.append(batch, k, v, rope=rope, q=q, q_out=q_out)
    out = cache.attention(batch, q_out)

A Batch8 holds addresses, so it serves every layer of a step and, as the
kernels read the arrays themselves, every later step that updates them in
place.  Calls go to torch's current stream unless one is given; what attention()
allocates by itself then belongs to that stream, as it does under
torch.cuda.stream().
"""
from __future__ import annotations

import torch
from torch import cuda as _cuda

from . import knapspec as ks

_BF16 = (torch.bfloat16,)
_KINDS = {torch.bfloat16: (ks.KS_DTYPE_BF16, _BF16), torch.float32: (ks.KS_DTYPE_F32, (torch.float32,))}


def _check(t, name: str, dtypes, ndim: int, device):
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name}: {t.dim()} dimensions, {ndim} expected")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, the cache is on {device}")


class Batch8:
    """The sequences of a call: page_table int32 [n_seqs, pages], row_offsets int32 [n_seqs + 1],
    lengths int32 [n_seqs] on the device; status: int32 [1] for what only the device can see.  Calls read the arrays
    while they run: update them in the calls' stream, or after them."""

    def __init__(self, page_table, row_offsets, lengths, n_rows: int, status=None):
        dev = page_table.device
        _check(page_table, "page_table", (torch.int32,), 2, dev)
        _check(row_offsets, "row_offsets", (torch.int32,), 1, dev)
        _check(lengths, "lengths", (torch.int32,), 1, dev)
        n = page_table.shape[0]
        if row_offsets.shape[0] != n + 1 or lengths.shape[0] != n:
            raise ValueError(f"{n} sequences, {row_offsets.shape[0]} offsets, {lengths.shape[0]} lengths")
        if n and page_table.stride(1) != 1 and page_table.shape[1] > 1:
            raise ValueError("page_table: a sequence's pages are not contiguous")
        if not (row_offsets.is_contiguous() and lengths.is_contiguous()):
            raise ValueError("row_offsets and lengths have to be contiguous")
        if n > 1 and page_table.stride(0) != page_table.shape[1]:
            raise ValueError("page_table: its rows are not one after the other")
        if status is not None:
            _check(status, "status", (torch.int32,), 1, dev)
            if status.numel() < 1:
                raise ValueError("status: no element")
        self._keep = (page_table, row_offsets, lengths, status)
        self.device, self.n_seqs, self.n_rows = dev, n, int(n_rows)
        self.c = ks.KsKv8Batch(ks._ptr(page_table), ks._ptr(row_offsets), ks._ptr(lengths), n, page_table.shape[1],
                               int(n_rows), ks._ptr(status))


class Cache8:
    """One layer's cache.  data: uint8, at least nbytes of it (allocated here if not given)."""

    def __init__(self, n_pages: int, page_tokens: int, n_kv_heads: int, head_dim: int, data=None, device="cuda"):
        self.nbytes = ks.ks_kv8_bytes(n_pages, page_tokens, n_kv_heads, head_dim)
        if self.nbytes == 0:
            raise ks.KsError(ks.KS_ERR_INVALID_ARG, "Cache8", f"sizes not supported: {n_pages} pages of {page_tokens} "
                             f"tokens, {n_kv_heads} heads of {head_dim}")
        if data is None:
            data = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        if data.dtype != torch.uint8 or not data.is_contiguous() or data.numel() < self.nbytes:
            raise ValueError(f"data: {self.nbytes} contiguous bytes expected")
        self.data, self.device = data, data.device
        self.n_kv_heads, self.head_dim = n_kv_heads, head_dim
        self.c = ks.KsKv8Cache(data.data_ptr(), n_pages, page_tokens, n_kv_heads, head_dim)

    def _stream(self, stream):
        index = _cuda.current_device()
        if self.device.index != index:
            raise ValueError(f"the cache is on {self.device}, not on the current device")
        if stream is None:
            # the address alone: torch.cuda.current_stream() builds an object in 2.8 us, a quarter of a small call
            return torch._C._cuda_getCurrentRawStream(index)
        if isinstance(stream, _cuda.Stream) and stream.device != self.device:
            raise ValueError(f"the cache is on {self.device}, the stream on {stream.device}")
        return ks._stream_ptr(stream)

    def _rows(self, t, name, kinds, batch, heads=None):
        """Row and head stride of a [rows, heads, head_dim] tensor, after its checks."""
        shape, stride = t.shape, t.stride()
        if (len(shape) != 3 or shape[2] != self.head_dim or shape[0] < batch.n_rows or t.dtype not in kinds or
                t.device != self.device or stride[2] != 1 or (heads is not None and shape[1] != heads)):
            _check(t, name, kinds, 3, self.device)
            raise ValueError(f"{name}: shape {tuple(shape)}, strides {stride} for {batch.n_rows} rows, "
                             f"{'any' if heads is None else heads} heads of {self.head_dim} contiguous values")
        return stride[0], stride[1]

    def append(self, batch: Batch8, k, v, rope=None, q=None, q_out=None, stream=None):
        """Append k, v [n_rows, n_kv_heads, head_dim] (fp32 or bf16); rope [positions, head_dim / 2, 2] fp32 rotates
        the keys, and the queries q [n_rows, n_q_heads, head_dim] into q_out (bf16)."""
        s = self._stream(stream)
        if batch.device != self.device:
            raise ValueError(f"the batch is on {batch.device}, the cache on {self.device}")
        code, kinds = _KINDS.get(k.dtype, (0, tuple(_KINDS)))
        k_row, k_head = self._rows(k, "k", kinds, batch, self.n_kv_heads)
        v_row, v_head = self._rows(v, "v", kinds, batch, self.n_kv_heads)
        angles, positions = None, 0
        if rope is not None:
            shape = rope.shape
            if rope.dtype != torch.float32 or rope.device != self.device or len(shape) != 3 or \
                    shape[1] != self.head_dim // 2 or shape[2] != 2 or not rope.is_contiguous():
                raise ValueError(f"rope: {rope.dtype} of shape {tuple(shape)} on {rope.device}")
            angles, positions = rope.data_ptr(), shape[0]
        if q is None and q_out is None:
            r = ks.KsKv8Rows(k.data_ptr(), v.data_ptr(), None, code, 0, k_row, k_head, v_row, v_head, 0, 0, angles,
                             positions)
        elif q is None or q_out is None:
            raise ValueError("q and q_out go together")
        else:
            q_row, q_head = self._rows(q, "q", kinds, batch)
            o_row, o_head = self._rows(q_out, "q_out", _BF16, batch, q.shape[1])
            r = ks.KsKv8Rows(k.data_ptr(), v.data_ptr(), q.data_ptr(), code, q.shape[1], k_row, k_head, v_row, v_head,
                             q_row, q_head, angles, positions, q_out.data_ptr(), o_row, o_head)
        ks.ks_kv8_append(self.c, batch.c, r, s)

    def read(self, batch: Batch8, k_out, v_out, stream=None):
        """The values of the batch's rows into k_out, v_out [n_rows, n_kv_heads, head_dim] (fp32 or bf16)."""
        s = self._stream(stream)
        if batch.device != self.device:
            raise ValueError(f"the batch is on {batch.device}, the cache on {self.device}")
        code, kinds = _KINDS.get(k_out.dtype, (0, tuple(_KINDS)))
        strides = self._rows(k_out, "k_out", kinds, batch, self.n_kv_heads)
        if self._rows(v_out, "v_out", kinds, batch, self.n_kv_heads) != strides:
            raise ValueError("k_out and v_out differ in their strides")
        ks.ks_kv8_read(self.c, batch.c, k_out.data_ptr(), v_out.data_ptr(), code, *strides, s)
        return k_out, v_out

    def attention_workspace(self, n_q_heads: int, n_seqs: int, n_rows: int):
        """A workspace of attention() for these sizes or smaller ones; calls that run at once need one each."""
        n = ks.ks_kv8_attention_workspace(self.c, n_q_heads, n_seqs, n_rows)
        if n == 0:
            raise ks.KsError(ks.KS_ERR_INVALID_ARG, "attention_workspace", f"{n_q_heads} query heads over "
                             f"{self.n_kv_heads}, {n_seqs} sequences, {n_rows} rows")
        return torch.empty(n, dtype=torch.uint8, device=self.device)

    def attention(self, batch: Batch8, q, scale=None, out=None, lse=None, workspace=None, stream=None):
        """Causal attention of the batch's rows: q, out [n_rows, n_q_heads, head_dim] bf16, lse [n_rows, n_q_heads]
        fp32.  scale: head_dim ** -0.5 if not given.  Returns out.  The address of a stream that is not the current
        one needs out and workspace with it: torch cannot allocate for an address."""
        s = self._stream(stream)
        if stream is not None and (out is None or workspace is None) and \
                s != torch._C._cuda_getCurrentRawStream(self.device.index):
            if not isinstance(stream, _cuda.Stream):
                raise ValueError("out and workspace: to be given with the address of a stream")
            # what the current stream allocates it may still write, the zeros below among it, and hand out again
            # while the call runs
            with _cuda.stream(stream):
                return self.attention(batch, q, scale, out, lse, workspace)
        if batch.device != self.device:
            raise ValueError(f"the batch is on {batch.device}, the cache on {self.device}")
        q_row, q_head = self._rows(q, "q", _BF16, batch)
        hq = q.shape[1]
        if out is None:
            out = torch.zeros(q.shape, dtype=torch.bfloat16, device=self.device)
        o_row, o_head = self._rows(out, "out", _BF16, batch, hq)
        sums = None
        if lse is not None:
            _check(lse, "lse", (torch.float32,), 2, self.device)
            if lse.shape[0] < batch.n_rows or lse.shape[1] != hq or not lse.is_contiguous():
                raise ValueError(f"lse: shape {tuple(lse.shape)}")
            sums = lse.data_ptr()
        if workspace is None:
            workspace = self.attention_workspace(hq, batch.n_seqs, batch.n_rows)
        elif workspace.device != self.device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous bytes on the cache's device expected")
        a = ks.KsKv8Attn(q.data_ptr(), q_row, q_head, out.data_ptr(), o_row, o_head, sums, hq,
                         self.head_dim ** -0.5 if scale is None else scale, workspace.data_ptr(), workspace.numel())
        ks.ks_kv8_attention(self.c, batch.c, a, s)
        return out
