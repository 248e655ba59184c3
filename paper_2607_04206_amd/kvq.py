"""Python face of the quantised KV cache (include/sangam_kvq.h): the attention
call of ``attn`` and the export and import of ``kv`` over pages of 8 or 4 bits a
value, with the plans of those modules. Argument marshalling only: every step
runs in the HIP kernels of libsangam_attn.so."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

from . import attn, kv
from ._lib import KvqCache, check, lib

# codes of a format: their C constant, dtype and dims per element
FORMATS = {"e4m3": (1, torch.float8_e4m3fn, 1), "e2m1": (2, torch.uint8, 2)}
BLOCK = 32  # consecutive dims of a row that share a scale


@dataclass(eq=False)
class QuantCache:
    """A pool of quantised pages. k, v: codes, torch.float8_e4m3fn [pages, Hkv,
    16, D] or, two e2m1 codes to a byte (the even dim in the low half),
    torch.uint8 [pages, Hkv, 16, D / 2]. k_scale, v_scale: torch.uint8 [pages,
    Hkv, 16, D / 32], the power of two b of a block standing for 2^(b - 127)
    (torch.float8_e8m0fnu shows them as numbers). The caller owns the tensors."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def __post_init__(self):
        if not isinstance(self.k, torch.Tensor):
            raise TypeError("k must be a torch.Tensor")
        by_dtype = {dtype: (name, per) for name, (_, dtype, per) in FORMATS.items()}
        if self.k.dtype not in by_dtype:
            raise TypeError(f"k must hold e4m3 codes (torch.float8_e4m3fn) or pairs of e2m1 codes (torch.uint8), got {self.k.dtype}")
        self.format, per = by_dtype[self.k.dtype]
        if self.k.dim() != 4 or self.k.shape[2] != 16 or self.k.shape[3] * per not in (64, 128):
            raise ValueError("k must be [num_pool_pages, Hkv, 16, D] with D 64 or 128 (e2m1: D / 2 bytes)")
        self.num_pool_pages, self.num_kv_heads = int(self.k.shape[0]), int(self.k.shape[1])
        self.head_dim = int(self.k.shape[3]) * per
        dev = self.k.device
        scales = tuple(self.k.shape[:3]) + (self.head_dim // BLOCK,)
        for t, name, dtype, shape in ((self.k, "k", self.k.dtype, tuple(self.k.shape)), (self.v, "v", self.k.dtype, tuple(self.k.shape)),
                                      (self.k_scale, "k_scale", torch.uint8, scales), (self.v_scale, "v_scale", torch.uint8, scales)):
            attn._need(t, name, dtype, shape, dev)

    def c_cache(self) -> KvqCache:
        return KvqCache(FORMATS[self.format][0], 0, self.num_pool_pages, self.k.data_ptr(), self.v.data_ptr(),
                        self.k_scale.data_ptr(), self.v_scale.data_ptr())


def empty_cache(num_pool_pages: int, num_kv_heads: int, head_dim: int, *, format: str = "e4m3", device=None) -> QuantCache:
    """A pool of that many pages, all zero."""
    if format not in FORMATS:
        raise ValueError(f"format must be one of {sorted(FORMATS)}, got {format!r}")
    if head_dim not in (64, 128):
        raise ValueError(f"head_dim must be 64 or 128, got {head_dim}")
    _, dtype, per = FORMATS[format]
    rows = (num_pool_pages, num_kv_heads, 16)
    codes = [torch.zeros(rows + (head_dim // per,), dtype=torch.uint8, device=device).view(dtype) for _ in range(2)]
    scales = [torch.zeros(rows + (head_dim // BLOCK,), dtype=torch.uint8, device=device) for _ in range(2)]
    return QuantCache(*codes, *scales)


def _expect(t: torch.Tensor, name: str, dtype, shape, dev) -> None:
    """attn._need's checks; its words where one fails."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.device == dev and t.is_contiguous()):
        attn._need(t, name, dtype, shape, dev)


def _launch(dev: torch.device, fn, *args) -> None:
    """The C call with dev as the current device."""
    if torch.cuda.current_device() == dev.index:
        check(fn(*args))
        return
    with torch.cuda.device(dev):
        check(fn(*args))


def _stream(dev: torch.device, stream: Optional[torch.cuda.Stream]) -> int:
    """The hipStream_t of the given or current stream (without a Stream object
    for the current one, which takes longer than the call's checks)."""
    if dev.type != "cuda":
        raise ValueError("the call needs device tensors (a ROCm GPU)")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev.index)
    if stream.device != dev:
        raise ValueError(f"stream belongs to {stream.device}, the tensors are on {dev}")
    return stream.cuda_stream


def _new(shape, dtype, dev, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A tensor that `stream`, if one was given, writes: of that stream's memory
    (the current stream may still work on what it has freed), not reused before
    what the current stream does with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=dev)
    t.record_stream(torch.cuda.current_stream(dev))
    return t


def _on_device(p, dev: torch.device, s: int, stream: Optional[torch.cuda.Stream]) -> int:
    """Address of the plan's copy on dev, made there if there is none; not
    reused before the call on stream `s` (the given or current one) has read it."""
    if p.dev is None or p.dev.device != dev:
        p.to(dev)
    if p.upload_stream is None or p.upload_stream.cuda_stream != s:
        p.dev.record_stream(stream if stream is not None else torch.cuda.current_stream(dev))
    return p.dev.data_ptr()


def forward(p: attn.Plan, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, cache: QuantCache,
            page_ids: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
            workspace: Optional[torch.Tensor] = None, want_lse: bool = True,
            stream: Optional[torch.cuda.Stream] = None,
            launch_events: Optional[Sequence[torch.cuda.Event]] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """sangam_kvq_forward on the current (or given) stream: attn.forward over a
    quantised cache, with a plan of attn.plan. The fresh rows are attended to as
    they are and written into the pages quantised."""
    dev = q.device
    s = _stream(dev, stream)
    T, Hq, Hkv, D = p.total_q, p.num_q_heads, p.num_kv_heads, p.head_dim
    _expect(q, "q", torch.bfloat16, (T, Hq, D), dev)
    _expect(k_new, "k_new", torch.bfloat16, (T, Hkv, D), dev)
    _expect(v_new, "v_new", torch.bfloat16, (T, Hkv, D), dev)
    _check_cache(cache, Hkv, D, p.num_pool_pages, dev)
    attn._need(page_ids, "page_ids", torch.int32, None, dev)
    num_page_ids = page_ids.numel()
    if page_ids.dim() != 1 or num_page_ids < p.total_pages:
        raise ValueError(f"page_ids must be a 1-D tensor of at least {p.total_pages} entries "
                         "(the plan's page table, on the device)")
    if out is not None:
        _expect(out, "out", torch.bfloat16, (T, Hq, D), dev)
    if lse is not None:
        _expect(lse, "lse", torch.float32, (T, Hq), dev)
    if workspace is not None and (not workspace.is_contiguous() or workspace.device != dev):
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    if launch_events is not None and len(launch_events) != 6:
        raise ValueError("launch_events needs 6 events (start and stop of 3 launches)")
    plan_dev = _on_device(p, dev, s, stream)
    if out is None:
        out = _new((T, Hq, D), torch.bfloat16, dev, stream)
    if lse is None and want_lse:
        lse = _new((T, Hq), torch.float32, dev, stream)
    if workspace is None and p.workspace_bytes > 0:
        workspace = _new((p.workspace_bytes,), torch.uint8, dev, stream)
    if p.upload_done is not None and p.upload_stream.cuda_stream != s:
        p.order_after_upload(stream if stream is not None else torch.cuda.current_stream(dev))
    evs = None if launch_events is None else (ctypes.c_void_p * 6)(*[e.cuda_event for e in launch_events])
    _launch(dev, lib.sangam_kvq_forward, p.host_ptr(), plan_dev, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
            ctypes.byref(cache.c_cache()), page_ids.data_ptr(), num_page_ids, out.data_ptr(),
            lse.data_ptr() if lse is not None else None, workspace.data_ptr() if workspace is not None else None,
            workspace.numel() * workspace.element_size() if workspace is not None else 0, s, evs)
    return out, lse


def _check_cache(cache: QuantCache, hkv: int, d: int, pages: int, dev) -> None:
    if not isinstance(cache, QuantCache):
        raise TypeError("cache must be a QuantCache")
    if cache.k.device != dev:
        raise ValueError(f"the cache must be on {dev}, got {cache.k.device}")
    if (cache.num_kv_heads, cache.head_dim) != (hkv, d):
        raise ValueError(f"the plan is for {hkv} KV heads of {d} dims, the cache holds {cache.num_kv_heads} of {cache.head_dim}")
    if cache.num_pool_pages < pages:
        raise ValueError(f"the plan addresses {pages} pool pages, the cache holds {cache.num_pool_pages}")


def _packed(p: kv.KvPlan, t: torch.Tensor, name: str, dev) -> None:
    """kv._check_packed's check; its words where it fails."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.device == dev and t.is_contiguous() and
            t.shape == (p.rows, p.num_kv_heads, p.head_dim)):
        kv._check_packed(p, t, name, dev)


def kv_export(p: kv.KvPlan, cache: QuantCache, k_packed: Optional[torch.Tensor] = None,
              v_packed: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """sangam_kvq_export on the current (or given) stream: the values of the
    listed requests' rows, bf16, with a plan of kv.plan. Allocates the packed
    buffers with torch when they are not passed."""
    dev = cache.k.device
    s = _stream(dev, stream)
    _check_cache(cache, p.num_kv_heads, p.head_dim, p.num_pool_pages, dev)
    shape = (p.rows, p.num_kv_heads, p.head_dim)
    if k_packed is None:
        k_packed = _new(shape, torch.bfloat16, dev, stream)
    if v_packed is None:
        v_packed = _new(shape, torch.bfloat16, dev, stream)
    _packed(p, k_packed, "k_packed", dev)
    _packed(p, v_packed, "v_packed", dev)
    _launch(dev, lib.sangam_kvq_export, p.host_ptr(), _on_device(p, dev, s, stream), ctypes.byref(cache.c_cache()), k_packed.data_ptr(),
            v_packed.data_ptr(), s)
    return k_packed, v_packed


def kv_import(p: kv.KvPlan, k_packed: torch.Tensor, v_packed: torch.Tensor, cache: QuantCache,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """sangam_kvq_import on the current (or given) stream: quantises the rows
    into the listed pages' slots [0, L_i) of the cache."""
    dev = cache.k.device
    s = _stream(dev, stream)
    _check_cache(cache, p.num_kv_heads, p.head_dim, p.num_pool_pages, dev)
    _packed(p, k_packed, "k_packed", dev)
    _packed(p, v_packed, "v_packed", dev)
    _launch(dev, lib.sangam_kvq_import, p.host_ptr(), _on_device(p, dev, s, stream), k_packed.data_ptr(), v_packed.data_ptr(),
            ctypes.byref(cache.c_cache()), s)
