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
from .kvq import _new, _stream

SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


@dataclass
class RopePlan:
    host: np.ndarray             # uint8 blob (host)
    dev: Optional[torch.Tensor]  # the same bytes on the device
    rot_dim: int
    interleaved: bool

    def host_ptr(self) -> int:
        return self.host.ctypes.data

    def to(self, device) -> "RopePlan":
        self.dev = torch.from_numpy(self.host).to(device)
        return self


def plan(*, rot_dim: int, interleaved: bool = False, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
         original_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: Optional[float] = None,
         device=None) -> RopePlan:
    """sangam_rope_plan: the rates of rot_dim / 2 pairs (host only). scaling:
    "none", "linear", "ntk" or "yarn", by `factor` beyond original_len
    positions; magnitude: the factor on cos and sin, by default the scaling's
    own. With ``device`` the blob is also copied to that device."""
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


def _check(t: torch.Tensor, name: str, rows: int, dtype, head_dim, device) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype or t.dtype not in DTYPES:
        raise TypeError(f"q and k must both be bfloat16, float16 or float32, got {t.dtype} for {name}")
    if t.dim() != 3 or t.shape[0] != rows or t.shape[1] < 1 or t.shape[2] != head_dim:
        raise ValueError(f"{name} must be [{rows}, heads, {head_dim}], got {tuple(t.shape)}")
    if t.stride(2) != 1:
        raise ValueError(f"the dims of a head of {name} must be consecutive")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two tensors [rows, heads, D] may share an element (exactly so for
    views that lie side by side in rows of one buffer)."""
    size = a.element_size()
    span = lambda t: sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1  # noqa: E731
    gap = (b.data_ptr() - a.data_ptr()) // size
    if gap >= span(a) or -gap >= span(b):
        return False
    row = a.stride(0)
    if a.shape[0] > 1 and row == b.stride(0) and row > 0:
        wa, wb = span(a[0]), span(b[0])
        at = gap % row
        if wa <= row and wb <= row and at >= wa and at + wb <= row:
            return False
    return True


def rotate(p: RopePlan, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, transpose: bool = False,
           stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """sangam_rope_rotate on the current (or given) stream: q [rows, Hq, D] and
    k [rows, Hkv, D] (or None), whose dims are consecutive and whose rows and
    heads may lie anywhere (views of a fused projection), rotated at positions,
    int32 [rows] on the device. Allocates the outputs with torch when they are
    not passed; q_out=q and k_out=k rotate in place. transpose gives the
    gradient with respect to q and k from that of the outputs."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise TypeError("q must be a torch.Tensor of three dimensions")
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    dev = q.device
    s = _stream(dev, stream)
    rows, d = int(q.shape[0]), int(q.shape[2])
    if not isinstance(positions, torch.Tensor) or positions.dtype != torch.int32:
        raise TypeError("positions must be an int32 tensor")
    if tuple(positions.shape) != (rows,) or not positions.is_contiguous() or positions.device != dev:
        raise ValueError(f"positions must be a contiguous [{rows}] tensor on {dev}")
    pairs = [(q, q_out, "q")] + ([(k, k_out, "k")] if k is not None else [])
    for t, o, name in pairs:
        _check(t, name, rows, q.dtype, d, dev)
        if o is not None:
            _check(o, name + "_out", rows, q.dtype, d, dev)
            if o.shape[1] != t.shape[1]:
                raise ValueError(f"{name}_out must have {t.shape[1]} heads, got {o.shape[1]}")
    if rows:
        outs = [o for _, o, _ in pairs if o is not None]
        for o in outs:
            for t, own, name in pairs:
                same = o is own and o.data_ptr() == t.data_ptr() and o.stride() == t.stride()
                if not same and _overlap(o, t):
                    raise ValueError(f"an output overlaps {name} without being it")
        if len(outs) == 2 and _overlap(*outs):
            raise ValueError("q_out and k_out overlap")
    with torch.cuda.device(dev):
        if p.dev is None or p.dev.device != dev:
            p.to(dev)
        done = [o if o is not None else _new(tuple(t.shape), t.dtype, dev, s) for t, o, _ in pairs]
        c = [RopeTensor(t.data_ptr(), o.data_ptr(), t.stride(0), t.stride(1), o.stride(0), o.stride(1), int(t.shape[1]), 0)
             for (t, _, _), o in zip(pairs, done)]
        check(lib.sangam_rope_rotate(p.host_ptr(), p.dev.data_ptr(), ctypes.byref(c[0]), ctypes.byref(c[1]) if k is not None else None,
                                     d, DTYPES[q.dtype], positions.data_ptr(), rows, int(bool(transpose)), s.cuda_stream))
    return done[0], done[1] if k is not None else None
