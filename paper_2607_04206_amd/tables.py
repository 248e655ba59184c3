"""Python face of the page tables (include/sangam_tables.h): block tables that
follow their requests' lengths, and what a batch's calls read of them, over
torch tensors. Argument marshalling only: both run in the HIP kernels of
libsangam_attn.so."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional

import torch

from ._lib import BlockTable, TablesBatch, lib
from .kvq import _launch, _new, _stream


MOST = 2 ** 31 - 1  # sizes are 32 bits to the C calls


@dataclass(eq=False)
class Tables:
    """What the calls of a batch read: page_indptr int32 [items + 1]; page_ids
    int32 [pages] (attn.forward); positions int32 [rows] (rope.rotate); slots
    int64 [rows] (sample.unmask), 16 page + position mod 16; items int32 [rows]
    (sample.tokens' params_of)."""
    page_indptr: torch.Tensor
    page_ids: torch.Tensor
    positions: torch.Tensor
    slots: torch.Tensor
    items: torch.Tensor


def _ints(t, name: str, dev, entries: Optional[int] = None, dtype=torch.int32) -> int:
    """Address of a contiguous tensor [entries] (None: of any) of that dtype on dev."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise TypeError(f"{name} must be a torch.Tensor of {dtype}")
    if t.get_device() != dev.index:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    if t.dim() != 1 or not t.is_contiguous() or (entries is not None and t.numel() != entries):
        raise ValueError(f"{name} must be a contiguous tensor [{'n' if entries is None else entries}], got {list(t.shape)}")
    return t.data_ptr()


def _table(table) -> BlockTable:
    if not isinstance(table, torch.Tensor) or table.dtype is not torch.int32 or table.dim() != 2:
        raise TypeError("table must be a torch.Tensor [requests, max_pages] of int32")
    requests, pages = table.shape
    if requests > MOST or pages > MOST:
        raise ValueError(f"table must have at most {MOST} requests and pages of a request, got {list(table.shape)}")
    if table.numel() and ((table.stride(1) != 1 and pages > 1) or (table.stride(0) < pages and requests > 1)):
        raise ValueError("the pages of a request must be consecutive, and requests apart")
    return BlockTable(table.data_ptr(), max(table.stride(0), pages) if requests > 1 else pages, requests, pages)


def resize(table: torch.Tensor, held: torch.Tensor, lengths: torch.Tensor, free: torch.Tensor, num_free: torch.Tensor,
           short: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """sangam_tables_resize on the current (or given) stream: every request of
    the table, int32 [requests, max_pages], gets exactly ceil(lengths / 16)
    pages; table, held (int32 [requests]), free (int32 [n], a stack of num_free
    pages) and num_free (int32 [1]) follow in place. Returns short, int32 [1]:
    how many requests found too few pages and got none."""
    c_table = _table(table)
    dev = table.device
    s = _stream(dev, stream)
    h = _ints(held, "held", dev, c_table.requests)
    n = _ints(lengths, "lengths", dev, c_table.requests)
    f = _ints(free, "free", dev)
    if free.numel() > MOST:
        raise ValueError(f"free must have at most {MOST} entries, got {free.numel()}")
    m = _ints(num_free, "num_free", dev, 1)
    if short is None:
        short = _new((1,), torch.int32, dev, stream)
        left = short.data_ptr()
    else:
        left = _ints(short, "short", dev, 1)
    _launch(dev, lib.sangam_tables_resize, ctypes.byref(c_table), h, n, f, free.numel(), m, left, s)
    return short


def build(table: torch.Tensor, request: Optional[torch.Tensor], kv_len: torch.Tensor, q_indptr: torch.Tensor, q_offset: torch.Tensor,
          *, rows: int, pages: int, q_pos: Optional[torch.Tensor] = None, out: Optional[Tables] = None,
          stream: Optional[torch.cuda.Stream] = None) -> Tables:
    """sangam_tables_build on the current (or given) stream: the page list,
    positions, slots and items of a batch's rows and pages, from the block table
    of its requests. Item i is request[i] (None: i), attends to kv_len[i]
    positions and has the rows q_indptr[i] to q_indptr[i + 1], from position
    q_offset[i] on or at q_pos. All int32 on the device; rows and pages are the
    sizes of what comes back, of which what no item has is padding (page -1,
    position 0, slot -1, item -1)."""
    c_table = _table(table)
    dev = table.device
    s = _stream(dev, stream)
    if rows < 0 or pages < 0:
        raise ValueError("rows and pages must not be negative")
    k = _ints(kv_len, "kv_len", dev)
    items = kv_len.numel()
    if items > MOST:
        raise ValueError(f"kv_len must have at most {MOST} entries, got {items}")
    batch = TablesBatch(items, 0, None if request is None else _ints(request, "request", dev, items), k,
                        _ints(q_indptr, "q_indptr", dev, items + 1), _ints(q_offset, "q_offset", dev, items),
                        None if q_pos is None else _ints(q_pos, "q_pos", dev, rows))
    if out is None:
        # (one allocation and no checks of it: each costs about as much as the launch's own work here)
        sizes = [2 * rows, rows, rows, items + 1, pages]
        memory = _new((sum(sizes),), torch.int32, dev, stream)
        slots, positions, row_items, page_indptr, page_ids = memory.split(sizes)
        out = Tables(page_indptr, page_ids, positions, slots.view(torch.int64), row_items)
        at = memory.data_ptr()
        to = at + 16 * rows, at + 16 * rows + 4 * (items + 1), at + 8 * rows, at, at + 12 * rows
    else:
        to = (_ints(out.page_indptr, "out.page_indptr", dev, items + 1), _ints(out.page_ids, "out.page_ids", dev, pages),
              _ints(out.positions, "out.positions", dev, rows), _ints(out.slots, "out.slots", dev, rows, torch.int64), _ints(out.items, "out.items", dev, rows))
    _launch(dev, lib.sangam_tables_build, ctypes.byref(c_table), ctypes.byref(batch), to[0], to[1], pages, to[2], to[3], to[4], rows, s)
    return out
