"""Python face of sampling and unmasking (include/sangam_sample.h): a token and a
confidence for every row of logits, and the rows of each block that take their
token, over torch tensors. Argument marshalling only: both run in the HIP
kernels of libsangam_attn.so."""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple, Union

import torch

from ._lib import SampleDesc, UnmaskDesc, lib
from .kvq import _launch, _new, _stream
from .rope import DTYPES
from .tables import MOST, _ints

CONFIDENCES = {"probability": 0, "margin": 1, "entropy": 2}
MAX_VOCAB = 1 << 18


def _each(x, name: str, dtype, dev, entries: Optional[int], lowest, highest):
    """A parameter as (address or None, value, entries): a tensor [entries] on dev, or a number."""
    if isinstance(x, torch.Tensor):
        return _ints(x, name, dev, entries, dtype), 0, x.numel()
    if not lowest <= x <= highest:
        raise ValueError(f"{name} must be {lowest} to {highest}, got {x}")
    return None, x, entries


def _result(t: Optional[torch.Tensor], name: str, entries: int, dtype, dev, stream) -> Tuple[torch.Tensor, int]:
    """The tensor that a result goes to, made here if none was passed, and its address."""
    if t is None:
        t = _new((entries,), dtype, dev, stream)
        return t, t.data_ptr()
    return t, _ints(t, name, dev, entries, dtype)


def tokens(logits: torch.Tensor, u: torch.Tensor, *, temperature: Union[float, torch.Tensor] = 1.0, top_k: Union[int, torch.Tensor] = 0,
           top_p: Union[float, torch.Tensor] = 1.0, min_p: Union[float, torch.Tensor] = 0.0, params_of: Optional[torch.Tensor] = None,
           confidence: str = "probability", forbid: int = -1, out: Optional[torch.Tensor] = None, confidence_out: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """sangam_sample_tokens on the current (or given) stream: a token (int32
    [rows]) and a confidence (float32 [rows]) for every row of logits [rows,
    vocab] (bfloat16, float16 or float32; rows may lie apart), by the uniform
    numbers u (float32 [rows], 0 to 1). The parameters are numbers, or tensors
    (float32, top_k int32) with an entry a row, or with params_of (int32 [rows])
    an entry a request: rows where params_of is outside get token -1. temperature
    0 takes the most likely token; top_k 0, top_p 1 and min_p 0 keep all.
    confidence: "probability" of the token, "margin" of the two most likely
    ones, or "entropy" (negative) of what is kept. forbid: a token that no row
    takes (the mask token), or -1."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in DTYPES:
        raise TypeError("logits must be a torch.Tensor [rows, vocab] of bfloat16, float16 or float32")
    if confidence not in CONFIDENCES:
        raise ValueError(f"confidence must be one of {sorted(CONFIDENCES)}, got {confidence!r}")
    dev = logits.device
    s = _stream(dev, stream)
    rows, vocab = logits.shape
    if not 1 <= vocab <= MAX_VOCAB:
        raise ValueError(f"vocab must be 1 to {MAX_VOCAB}, got {vocab}")
    if logits.stride(1) != 1 and vocab > 1 and rows > 0:
        raise ValueError("the logits of a row must be consecutive")
    if not -1 <= forbid < vocab:
        raise ValueError(f"forbid must be -1 or a token, got {forbid}")
    of = None if params_of is None else _ints(params_of, "params_of", dev, rows)
    entries = rows if params_of is None else None
    t, t_all, entries = _each(temperature, "temperature", torch.float32, dev, entries, 0.0, math.inf)
    k, k_all, entries = _each(top_k, "top_k", torch.int32, dev, entries, 0, 2 ** 31 - 1)
    p, p_all, entries = _each(top_p, "top_p", torch.float32, dev, entries, 0.0, 1.0)
    m, m_all, entries = _each(min_p, "min_p", torch.float32, dev, entries, 0.0, 1.0)
    out, to = _result(out, "out", rows, torch.int32, dev, stream)
    confidence_out, c_to = _result(confidence_out, "confidence_out", rows, torch.float32, dev, stream)
    dtype = DTYPES[logits.dtype]
    need = lib.sangam_sample_workspace_bytes(rows, vocab, dtype)
    if workspace is None and need > 0:
        workspace = _new((need,), torch.uint8, dev, stream)
    elif workspace is not None and (not workspace.is_contiguous() or workspace.device != dev):
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    d = SampleDesc(logits.data_ptr(), rows, logits.stride(0) if rows > 1 else 0, vocab, dtype, _ints(u, "u", dev, rows, torch.float32), of,
                   2 ** 31 if entries is None else entries, t, k, p, m, t_all, k_all, p_all, m_all, CONFIDENCES[confidence], forbid)
    _launch(dev, lib.sangam_sample_tokens, ctypes.byref(d), to, c_to, workspace.data_ptr() if workspace is not None else None,
            workspace.numel() * workspace.element_size() if workspace is not None else 0, s)
    return out, confidence_out


def unmask(tokens: torch.Tensor, confidence: torch.Tensor, ids: torch.Tensor, row_indptr: torch.Tensor, *, mask_id: int,
           count: Union[int, torch.Tensor] = 1, threshold: Union[float, torch.Tensor] = math.inf, slots: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, left: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """sangam_sample_unmask on the current (or given) stream: of every block (rows
    row_indptr[i] to row_indptr[i + 1]) the masked rows whose confidence is at
    least threshold, and the `count` most confident ones, take their token. tokens
    (int32) and confidence (float32) as sample.tokens gives them; ids: int32
    [rows], or with slots (int64 [rows], of tables.build) the pool [16 pages] that
    they address, where taken tokens are written. count and threshold: numbers, or
    tensors with an entry a block (int32, float32). Returns the rows' ids after
    the step (int32 [rows]; out=ids writes them in place) and how many of each
    block are still masked (int32 [blocks])."""
    if not isinstance(tokens, torch.Tensor) or tokens.dim() != 1 or tokens.dtype is not torch.int32:
        raise TypeError("tokens must be a torch.Tensor [rows] of int32")
    dev, rows = tokens.device, tokens.shape[0]
    s = _stream(dev, stream)
    indptr = _ints(row_indptr, "row_indptr", dev)
    blocks = row_indptr.shape[0] - 1
    if not 0 <= blocks <= MOST:
        raise ValueError(f"row_indptr must hold an entry more than blocks, which are at most {MOST}")
    if not -MOST - 1 <= mask_id <= MOST:
        raise ValueError(f"mask_id must fit 32 bits, got {mask_id}")
    n, n_all, _ = _each(count, "count", torch.int32, dev, blocks, 0, 2 ** 31 - 1)
    c, c_all, _ = _each(threshold, "threshold", torch.float32, dev, blocks, -math.inf, math.inf)
    out, to = _result(out, "out", rows, torch.int32, dev, stream)
    left, l_to = _result(left, "left", blocks, torch.int32, dev, stream)
    d = UnmaskDesc(_ints(tokens, "tokens", dev, rows),
                   _ints(confidence, "confidence", dev, rows, torch.float32), _ints(ids, "ids", dev, rows if slots is None else None),
                   None if slots is None else _ints(slots, "slots", dev, rows, torch.int64), indptr, n, c, rows, ids.shape[0], blocks,
                   mask_id, n_all, c_all)
    _launch(dev, lib.sangam_sample_unmask, ctypes.byref(d), to, l_to, s)
    return out, left
