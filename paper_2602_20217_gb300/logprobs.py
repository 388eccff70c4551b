"""Python face of ks_token_logprobs (include/knapspec.h): torch allocates the
memory, this module checks the tensors and marshals their addresses; the work
runs in the library's CUDA kernels.

    got = token_logprobs(logits, tokens, n_top=20)
    got.logprobs, got.entropy, got.top_ids, got.top_logprobs
"""
from __future__ import annotations

from typing import NamedTuple

import torch
from torch import cuda as _cuda

from . import knapspec as ks

_KINDS = {torch.bfloat16: ks.KS_DTYPE_BF16, torch.float32: ks.KS_DTYPE_F32}


class LogProbs(NamedTuple):
    """logprobs [rows, n] fp32, entropy [rows] fp32, top_ids [rows, n_top] int32, top_logprobs [rows, n_top] fp32."""
    logprobs: object
    entropy: object
    top_ids: object
    top_logprobs: object


def empty(rows: int, n_tokens: int, n_top: int, device="cuda") -> LogProbs:
    """Results to fill: a serving loop makes them once."""
    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=device)
    return LogProbs(new(rows, n_tokens), new(rows), new(rows, n_top, dtype=torch.int32), new(rows, n_top))


def marshal(logits, code: int, vocab: int, stride: int, tokens, n_top: int, temperature: float, out: LogProbs):
    """The library's form of a call, after the checks of tokens [rows, n] and of the results."""
    rows, n = tokens.shape
    device = tokens.device
    if tokens.dtype != torch.int32 or not tokens.is_contiguous():
        raise ValueError(f"tokens: {tokens.dtype}, strides {tokens.stride()}; contiguous int32 expected")
    for name, t, shape, dtype in (("logprobs", out.logprobs, (rows, n), torch.float32),
                                  ("entropy", out.entropy, (rows,), torch.float32),
                                  ("top_ids", out.top_ids, (rows, n_top), torch.int32),
                                  ("top_logprobs", out.top_logprobs, (rows, n_top), torch.float32)):
        if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
            raise ValueError(f"{name}: {t.dtype} of shape {tuple(t.shape)} on {t.device}; contiguous {dtype} of shape "
                             f"{shape} on {device} expected")
    return ks.KsLogprobs(logits, code, rows, vocab, stride, tokens.data_ptr(), n, n_top, temperature,
                         out.logprobs.data_ptr(), out.entropy.data_ptr(), out.top_ids.data_ptr(),
                         out.top_logprobs.data_ptr())


def token_logprobs(logits, tokens, n_top: int = 0, temperature: float = 1.0, out: LogProbs | None = None,
                   stream=None) -> LogProbs:
    """Log probabilities of tokens [rows] or [rows, n] (int32) under logits [rows, vocab] (fp32 or bf16, rows any
    distance apart), the rows' entropies and n_top largest logits.  out: the results of empty(rows, n, n_top), n being 1
    for tokens [rows].  Calls go to torch's current stream unless one is given; with the address of a stream that is not
    the current one the results have to be given."""
    index = _cuda.current_device()
    device = logits.device
    if device.type != "cuda" or device.index != index:
        raise ValueError(f"logits: on {device}, not on the current device")
    code = _KINDS.get(logits.dtype)
    if code is None or logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError(f"logits: {logits.dtype} of shape {tuple(logits.shape)}, strides {logits.stride()}; fp32 or bf16 "
                         "rows of contiguous values expected")
    if tokens.device != device or tokens.dim() not in (1, 2) or tokens.shape[0] != logits.shape[0]:
        raise ValueError(f"tokens: shape {tuple(tokens.shape)} on {tokens.device} for {logits.shape[0]} rows on {device}")
    if isinstance(stream, _cuda.Stream) and stream.device != device:
        raise ValueError(f"logits: on {device}, the stream on {stream.device}")
    current = torch._C._cuda_getCurrentRawStream(index)
    s = current if stream is None else ks._stream_ptr(stream)
    t = tokens if tokens.dim() == 2 else tokens[:, None]
    if out is None:
        if s != current:
            if not isinstance(stream, _cuda.Stream):
                raise ValueError("out: to be given with the address of a stream")
            with _cuda.stream(stream):
                out = empty(*t.shape, n_top, device=device)
        else:
            out = empty(*t.shape, n_top, device=device)
    ks.ks_token_logprobs(marshal(logits.data_ptr(), code, logits.shape[1], logits.stride(0), t, n_top, temperature,
                                 out), s)
    return out
