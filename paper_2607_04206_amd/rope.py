"""Python face of rotary positions (include/sangam_rope.h): plan and rotate over
torch tensors. Argument marshalling only: the rotation runs in the HIP kernels
of libsangam_attn.so."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional, Tuple

import numpy as np
import torch

from . import _lib
from ._lib import RopeDesc, RopeTensor, check, lib
from .kvq import _launch, _new, _on_device, _stream

SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "yarn_index": 4}
DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


@dataclass
class RopePlan:
    host: np.ndarray             # uint8 blob (host)
    dev: Optional[torch.Tensor]  # the same bytes on the device
    rot_dim: int
    interleaved: bool
    upload_stream: Optional[torch.cuda.Stream] = None  # the stream the device copy was made on

    def __post_init__(self):
        self._ptr = self.host.ctypes.data

    def host_ptr(self) -> int:
        return self._ptr

    def to(self, device) -> "RopePlan":
        self.dev = torch.from_numpy(self.host).to(device)
        self.upload_stream = torch.cuda.current_stream(self.dev.device) if self.dev.is_cuda else None
        return self


def plan(*, rot_dim: int, interleaved: bool = False, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
         original_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: Optional[float] = None,
         device=None) -> RopePlan:
    """sangam_rope_plan: the rates of rot_dim / 2 pairs (host only). scaling:
    "none", "linear", "ntk", "yarn" or "yarn_index", by `factor` beyond
    original_len positions; magnitude: the factor on cos and sin, by default the
    scaling's own. "yarn" is the paper's ramp, in the turns of a pair;
    checkpoints released with YaRN scaling take "yarn_index", in its index. With
    ``device`` the blob is also copied to that device."""
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(SCALINGS)}, got {scaling!r}")
    if magnitude is not None and not magnitude > 0:
        raise ValueError(f"magnitude must be positive, got {magnitude}")
    d = RopeDesc(int(rot_dim), int(bool(interleaved)), SCALINGS[scaling], 0, float(base), float(factor), float(original_len),
                 float(beta_fast), float(beta_slow), float(magnitude or 0.0))
    used = ctypes.c_size_t(0)
    st = lib.sangam_rope_plan(ctypes.byref(d), None, 0, ctypes.byref(used))
    if st not in (_lib.SANGAM_OK, -5):  # -5: buffer too small, *used holds the size
        check(st)
    buf = np.zeros(int(used.value), np.uint8)
    check(lib.sangam_rope_plan(ctypes.byref(d), buf.ctypes.data, buf.nbytes, ctypes.byref(used)))
    p = RopePlan(host=buf, dev=None, rot_dim=int(rot_dim), interleaved=bool(interleaved))
    if device is not None:
        p.to(device)
    return p


def _expect(t: torch.Tensor, name: str, shape, dtype, dev) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} as q is, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")


def _tensor(t: torch.Tensor, out: torch.Tensor, name: str, heads: int) -> RopeTensor:
    (row, head, dim), (out_row, out_head, out_dim) = t.stride(), out.stride()
    if (dim != 1 or out_dim != 1) and t.shape[2] > 1 and t.numel() > 0:
        raise ValueError(f"the dims of a head of {name} and of its output must be consecutive")
    return RopeTensor(t.data_ptr(), out.data_ptr(), row, head, out_row, out_head, heads, 0)


class _Rotate(torch.autograd.Function):
    """rotate for inputs that require gradients, which the transpose gives."""

    @staticmethod
    def forward(ctx, q, k, positions, p, transpose, stream):
        out = rotate(p, q, k, positions, transpose=transpose, stream=stream)
        ctx.save_for_backward(positions)
        ctx.plan, ctx.transpose = p, transpose
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(y for x, y in zip((q, k), out) if x is not None and not x.requires_grad))
        return out

    @staticmethod
    def backward(ctx, *grads):
        # (on the current stream, on which autograd orders both ends)
        positions, = ctx.saved_tensors
        need = [g is not None and n for g, n in zip(grads, ctx.needs_input_grad)]
        grads = [(g if g.stride(-1) == 1 else g.contiguous()) for g, n in zip(grads, need) if n]
        got = iter(rotate(ctx.plan, grads[0], grads[1] if len(grads) > 1 else None, positions, transpose=not ctx.transpose) if grads else ())
        return (*(next(got) if n else None for n in need), None, None, None, None)


def rotate(p: RopePlan, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, transpose: bool = False,
           stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """sangam_rope_rotate on the current (or given) stream: q [rows, Hq, D] and
    k [rows, Hkv, D] (or None), whose dims are consecutive and whose rows and
    heads may lie anywhere (views of a fused projection), rotated at positions,
    int32 [rows] on the device. Allocates the outputs with torch when they are
    not passed; q_out=q and k_out=k rotate in place. transpose gives the
    gradient with respect to q and k from that of the outputs. Where q or k
    requires gradients (and they are enabled), autograd gets them so; outputs
    that are passed are then refused, as nothing would record them."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in DTYPES:
        raise TypeError("q must be a torch.Tensor [rows, heads, D] of bfloat16, float16 or float32")
    dev, dtype = q.device, q.dtype
    s = _stream(dev, stream)
    if torch.is_grad_enabled() and (q.requires_grad or (isinstance(k, torch.Tensor) and k.requires_grad)):
        if q_out is not None or k_out is not None:
            raise ValueError("q_out and k_out record no gradients, which q or k requires: pass neither, or call under torch.no_grad()")
        return _Rotate.apply(q, k, positions, p, transpose, stream)
    rows, heads, d = q.shape
    if not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32:
        raise TypeError("positions must be an int32 tensor")
    if positions.shape != (rows,) or not positions.is_contiguous() or positions.device != dev:
        raise ValueError(f"positions must be a contiguous [{rows}] tensor on {dev}")
    if q_out is None:
        q_out = _new(q.shape, dtype, dev, stream)
    else:
        _expect(q_out, "q_out", q.shape, dtype, dev)
    c_q, c_k = _tensor(q, q_out, "q", heads), None
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            raise TypeError("k must be a torch.Tensor [rows, heads, D]")
        kv_heads = k.shape[1]
        _expect(k, "k", (rows, kv_heads, d), dtype, dev)
        if k_out is None:
            k_out = _new(k.shape, dtype, dev, stream)
        else:
            _expect(k_out, "k_out", k.shape, dtype, dev)
        c_k = ctypes.byref(_tensor(k, k_out, "k", kv_heads))
    elif k_out is not None:
        raise ValueError("k_out without k")
    _launch(dev, lib.sangam_rope_rotate, p.host_ptr(), _on_device(p, dev, s, stream), ctypes.byref(c_q), c_k, d, DTYPES[dtype],
            positions.data_ptr(), rows, 1 if transpose else 0, s)
    return q_out, k_out
