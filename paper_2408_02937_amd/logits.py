"""Binding of include/rtams_logits.h: log probabilities of given tokens, entropy and the most likely tokens of rows of logits.

Argument marshalling only: every step runs in the HIP kernels behind the C ABI, calls are asynchronous on the stream given (the current
one unless told), there is no fallback.  Tensors handed to a call on a stream given are kept for that stream.  Nothing here has a
gradient, and logits that ask for one are refused.

    s = score(logits, tokens, top=5)                # logits [rows][vocab], tokens int32 [rows] or [rows][m]
    s.logprobs, s.entropy, s.top, s.top_logprobs    # [rows][m], [rows], [rows][5] (tokens), [rows][5]
"""
from __future__ import annotations

import struct
from contextlib import nullcontext
from ctypes import sizeof
from typing import NamedTuple, Optional

import torch

from paper_2408_02937_amd.rtams import LogitsQuery, _chk, lib

_FORMAT = "@qqiiiifPPPPPPPPN"
_query = struct.Struct(_FORMAT).pack  # LogitsQuery
assert struct.calcsize(_FORMAT) == sizeof(LogitsQuery)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_MANY = 1024  # rows: of so many or more no call takes scratch,
_ONE = 65_520  # nor of rows of so many bytes


class Scores(NamedTuple):
    lse: torch.Tensor                      # [rows] logarithm of the sum of exp(scale * logit)
    entropy: torch.Tensor                  # [rows]
    logprobs: Optional[torch.Tensor]       # [rows][m] of the tokens given ([rows] where they are [rows])
    top: Optional[torch.Tensor]            # [rows][top] int32: the most likely tokens, -1 where there are no more
    top_logprobs: Optional[torch.Tensor]   # [rows][top]


def score(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, scale: float = 1.0, stream=None) -> Scores:
    """What rows of logits, bfloat16, float16 or float32 [rows][vocab], say of the tokens given and of all; scale: the inverse of a temperature.
    Equally likely tokens come lowest first.  A logit of -inf is a token that is not allowed."""
    if not (logits.dim() == 2 and logits.is_cuda and logits.dtype in _TYPES and logits.shape[1] > 0 and (logits.stride(1) == 1 or logits.shape[1] == 1)):
        raise ValueError("logits must be a bfloat16, float16 or float32 CUDA tensor [rows][vocab] whose rows' logits lie next to each other")
    if logits.requires_grad and torch.is_grad_enabled():
        raise ValueError("logits ask for a gradient, which score does not have: detach them, or call under torch.no_grad()")
    rows, vocab = logits.shape
    device = logits.device
    given = 0
    if tokens is not None:
        if not (tokens.dtype == torch.int32 and tokens.dim() in (1, 2) and tokens.shape[0] == rows and tokens.is_contiguous() and tokens.device == device):
            raise ValueError(f"tokens must be a contiguous int32 tensor [rows] or [rows][m] on {device}")
        given = tokens.shape[1] if tokens.dim() == 2 else 1
    if top < 0 or top > 64:
        raise ValueError("top must be in 0..64")
    if stream is not None:
        with torch.cuda.stream(stream):
            made = _outputs(rows, given, top, device)
    else:
        made = _outputs(rows, given, top, device)
    lse, entropy, logprobs, top_logprobs, best = made
    fields = (rows, logits.stride(0), vocab, _TYPES[logits.dtype], top, given, scale, logits.data_ptr(), tokens.data_ptr() if given else 0, lse.data_ptr(),
              entropy.data_ptr(), logprobs.data_ptr() if given else 0, best.data_ptr() if top else 0, top_logprobs.data_ptr() if top else 0)
    L = lib()
    at = size = 0
    if rows < _MANY and vocab * logits.element_size() > _ONE:
        size = L.rtams_logits_scratch_bytes_for(_query(*fields, 0, 0))
        if 0 < size < 1 << 62:
            with nullcontext() if stream is None else torch.cuda.stream(stream):
                scratch = torch.empty(size, dtype=torch.uint8, device=device)  # (the allocator hands it to later work of this stream only)
            at = scratch.data_ptr()
        else:
            size = 0
    if stream is None:
        pointer = _current_stream(device.index)
    else:
        pointer = stream.cuda_stream
        for t in (logits, tokens):
            if t is not None:
                t.record_stream(stream)
        now = torch.cuda.current_stream(device)
        for t in (lse, best):  # (the others are views of the first)
            if t is not None:
                t.record_stream(now)
    query = _query(*fields, at, size)
    if torch.cuda.current_device() == device.index:
        _chk(L.rtams_logits_score(query, pointer), "rtams_logits_score")
    else:
        with torch.cuda.device(device):
            _chk(L.rtams_logits_score(query, pointer), "rtams_logits_score")
    if tokens is not None and logprobs.shape != tokens.shape:
        logprobs = logprobs.view(tokens.shape)
    return Scores(lse, entropy, logprobs if tokens is not None else None, best, top_logprobs)


def _outputs(rows: int, given: int, top: int, device):
    """(lse, entropy, logprobs, top_logprobs, top): views of one tensor, and one for the tokens."""
    out = torch.empty(rows * (2 + given + top), dtype=torch.float32, device=device)
    lse, entropy, logprobs, top_logprobs = out.split_with_sizes((rows, rows, rows * given, rows * top))
    if top == 0:
        return lse, entropy, logprobs, None, None
    return lse, entropy, logprobs, top_logprobs.view(rows, top), torch.empty((rows, top), dtype=torch.int32, device=device)
