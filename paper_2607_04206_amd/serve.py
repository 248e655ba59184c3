"""A serving loop around the attention call: requests move through the
cached-dLLM cycle (whole prefill of prompt + masked response, then block
decodes of one 32-token block until it is resolved, then a re-prefill that
refreshes the cache at the block boundary; Sec. 2.2, Sec. 4.3), each
iteration's microbatch is composed by the deficit token-budget rule
(Sec. 4.1, Alg. 1) and served by one sangam_attn_forward call over a paged KV
pool (Sec. 5), or by one sangam_kvq_forward call over a quantised pool. With
rotary positions, q and k are rotated at their rows' positions before it. With
sampling, each decode row takes a token from logits (sample.tokens), and the most
confident rows of each block keep theirs (sample.unmask), which decides how many
steps a block takes; the block table then lies on the device and follows the
requests' lengths (tables.resize), and each batch's page list, positions and slots
are built there (tables.build). Without it the slots are not read, and the host
sends the page list and positions that it has.

Only one attention layer is run per iteration (the model around it is out of
scope), with synthetic Q / K / V values and logits: the loop exercises batch
composition, planning and the kernels on real mixed batches."""
from __future__ import annotations

import dataclasses
import time
from typing import List, Optional

import numpy as np
import torch

from . import attn, kv, kvq, rope, sample, sched, tables

BLOCK = 32
PAGE = 16


class PagePool:
    """Free list of KV pages of one pool (host side)."""

    def __init__(self, num_pages: int):
        self.num_pages = num_pages
        self._free = list(range(num_pages - 1, -1, -1))

    def take(self, n: int) -> List[int]:
        if n > len(self._free):
            raise MemoryError(f"KV pool exhausted: {n} pages wanted, {len(self._free)} free")
        return [self._free.pop() for _ in range(n)]

    def give(self, pages: List[int]) -> None:
        self._free.extend(reversed(pages))

    @property
    def free(self) -> int:
        return len(self._free)


@dataclasses.dataclass
class _State:
    req: object                 # workloads.TraceRequest
    pages: Optional[List[int]] = None
    block: int = 0              # block being decoded (or to decode after the prefill)
    steps_left: int = 0
    phase: str = "waiting"      # waiting (for a prefill), decoding, done
    queued_at: int = 0
    fresh: bool = False         # its response has no ids yet

    @property
    def L(self) -> int:
        return self.req.prompt + self.req.resp


@dataclasses.dataclass
class Iteration:
    t: int
    decodes: int
    prefills: int
    prefill_tokens: int
    waiting_after: int
    deficit: int
    plan_ms: float
    events: Optional[tuple] = None  # (start, end) torch events around the call
    # start / stop events in the dispatch of each launch that ran (prefill-
    # shaped, decode-shaped, merge): kernel execution without host gaps
    launch_events: Optional[list] = None
    queue_waits: List[int] = dataclasses.field(default_factory=list)
    captured: Optional[dict] = None
    batch: Optional[list] = None  # (request id, kind) of each item, in batch order
    left: Optional[List[int]] = None  # with sampling: rows of each decode's block that are still masked


class ServingLoop:
    """Drive a list of trace requests through iterations of one GPU.

    kv_format: None for a bf16 cache, or a format of kvq.FORMATS.
    rotary: None, or the arguments of rope.plan (rot_dim is the head dim unless
    they say otherwise).
    sampling: None (blocks take the trace's steps), or vocab, and any of
    temperature, top_k, top_p, min_p and confidence of sample.tokens and of count
    and threshold (0.9, the paper's) of sample.unmask: a block is done when no row
    of it is masked. Token vocab is the mask."""

    def __init__(self, requests, *, hq: int, hkv: int, d: int, tau: int, device,
                 num_pool_pages: Optional[int] = None, max_rows: int = 1 << 15, seed: int = 0,
                 kv_format: Optional[str] = None, rotary: Optional[dict] = None, sampling: Optional[dict] = None):
        if kv_format is not None and kv_format not in kvq.FORMATS:
            raise ValueError(f"kv_format must be None or one of {sorted(kvq.FORMATS)}, got {kv_format!r}")
        self.reqs = [_State(r) for r in sorted(requests, key=lambda r: (r.arrival, r.rid))]
        self.hq, self.hkv, self.d, self.tau = hq, hkv, d, tau
        self.dev = device
        need = sum(-(-(s.L) // PAGE) for s in self.reqs)
        self.pool = PagePool(num_pool_pages if num_pool_pages is not None else max(need, 1))
        self.max_rows = max_rows
        self.rope = None if rotary is None else rope.plan(**{"rot_dim": d, **rotary}, device=device)
        self.cache = None  # the quantised pool
        if device is not None:  # device None: plan every batch but run nothing (host checks)
            g = torch.Generator(device="cpu").manual_seed(seed)
            shape = (self.pool.num_pages, hkv, PAGE, d)
            self.k_cache = torch.randn(shape, generator=g).to(torch.bfloat16).to(device)
            self.v_cache = torch.randn(shape, generator=g).to(torch.bfloat16).to(device)
            self.q = torch.randn((max_rows, hq, d), generator=g).to(torch.bfloat16).to(device)
            self.k_new = torch.randn((max_rows, hkv, d), generator=g).to(torch.bfloat16).to(device)
            self.v_new = torch.randn((max_rows, hkv, d), generator=g).to(torch.bfloat16).to(device)
            if kv_format is not None:
                self._quantise_pool(kv_format)
            if self.rope is not None:
                self.q_rot, self.k_rot = torch.empty_like(self.q), torch.empty_like(self.k_new)
            self.out = torch.empty((max_rows, hq, d), dtype=torch.bfloat16, device=device)
            self.lse = torch.empty((max_rows, hq), dtype=torch.float32, device=device)
            # the block table follows the requests' lengths (0 before the first prefill and after the end)
            self._rows = {id(s): i for i, s in enumerate(self.reqs)}
            self.table = torch.full((len(self.reqs), max([-(-s.L // PAGE) for s in self.reqs], default=0)), -1, dtype=torch.int32, device=device)
            self.held = torch.zeros(len(self.reqs), dtype=torch.int32, device=device)
            self.free_pages = torch.tensor(self.pool._free, dtype=torch.int32, device=device)
            self.num_free = torch.tensor([self.pool.free], dtype=torch.int32, device=device)
            self._lengths = np.zeros(len(self.reqs), np.int32)
            self._changes = [[]]  # of the lengths, (request, length) by iteration, that the table does not follow yet
            self._short = []  # requests that the table had no pages for, of each change: not looked at yet
        self.sampling = None
        if sampling is not None:
            self._set_sampling(device, seed, **sampling)
        self.deficit = 0
        self.next_arrival = 0
        self.waiting: List[_State] = []  # arrival order of the requests (re-prefills keep their place)
        self.sm_scale = float(np.float32(1.0 / np.sqrt(d)))

    def _set_sampling(self, device, seed, *, vocab: int, count: int = 1, threshold: float = 0.9, **how) -> None:
        if not 1 <= vocab < sample.MAX_VOCAB:
            raise ValueError(f"vocab must be 1 to {sample.MAX_VOCAB - 1}, got {vocab}")
        if count < 1:
            raise ValueError("count must be 1 at least: a block of no confident row would not end")
        unknown = set(how) - {"temperature", "top_k", "top_p", "min_p", "confidence"}
        if unknown:
            raise ValueError(f"sampling does not take {sorted(unknown)}")
        self.sampling, self.mask_id = {"temperature": 0.0, **how}, vocab
        self.count, self.threshold = count, threshold
        if device is None:
            return
        self._gen = torch.Generator(device=device).manual_seed(seed)
        # one token id a slot of the pool, and a step's logits, the mask's own included (that no row takes)
        self.ids = torch.full((PAGE * self.pool.num_pages,), -1, dtype=torch.int32, device=device)
        self.logits = torch.empty((0, vocab + 1), dtype=torch.bfloat16, device=device)

    def _page_rows(self, page_ids: np.ndarray) -> kv.KvPlan:
        """A plan of all rows of some pages."""
        n = len(page_ids)
        return kv.plan(kv_len=[PAGE * n], page_indptr=[0, n], page_ids=page_ids, num_kv_heads=self.hkv, head_dim=self.d,
                       num_pool_pages=self.pool.num_pages, device=self.dev)

    def _quantise_pool(self, kv_format: str) -> None:
        """The bf16 pool's content in quantised pages, in its place."""
        p = self._page_rows(np.arange(self.pool.num_pages, dtype=np.int32))
        self.cache = kvq.empty_cache(self.pool.num_pages, self.hkv, self.d, format=kv_format, device=self.dev)
        kvq.kv_import(p, *kv.kv_export(p, self.k_cache, self.v_cache), self.cache)
        self.k_cache = self.v_cache = None

    def _pages(self, page_ids: np.ndarray, pid: torch.Tensor):
        """Copies of some pages' K and V, bf16 [pages, Hkv, 16, D]."""
        if self.cache is None:
            return self.k_cache[pid.long()].clone(), self.v_cache[pid.long()].clone()
        rows = kvq.kv_export(self._page_rows(page_ids), self.cache)
        return tuple(x.view(-1, PAGE, self.hkv, self.d).transpose(1, 2).contiguous() for x in rows)

    def _arrive(self, t: int) -> None:
        while self.next_arrival < len(self.reqs) and self.reqs[self.next_arrival].req.arrival <= t:
            s = self.reqs[self.next_arrival]
            s.queued_at = t
            self.waiting.append(s)
            self.next_arrival += 1
        self.waiting.sort(key=lambda s: (s.req.arrival, s.req.rid))

    def busy(self) -> bool:
        return self.next_arrival < len(self.reqs) or any(s.phase != "done" for s in self.reqs)

    def step(self, t: int, timed: bool = True, capture: bool = False) -> Optional[Iteration]:
        """One iteration: compose the microbatch, run the call, advance states.
        capture: keep the call's descriptor and a copy of its inputs (the
        pages' pre-call content included) on the record, for checking."""
        self._arrive(t)
        decodes = [s for s in self.reqs if s.phase == "decoding"]
        n_adm, self.deficit = sched.admit(self.tau, BLOCK * len(decodes), len(decodes),
                                          [s.L for s in self.waiting], self.deficit)
        admitted = self.waiting[:n_adm]
        del self.waiting[:n_adm]
        if not decodes and not admitted:
            return None
        for s in admitted:
            if s.pages is None:  # a request's pages live from its first prefill to its end
                s.pages = self.pool.take(-(-s.L // PAGE))
                s.fresh = True
                self._resize(s, s.L)
        items = decodes + admitted
        nd = len(decodes)
        n = [BLOCK] * nd + [s.L for s in admitted]
        o = [s.req.prompt + BLOCK * s.block for s in decodes] + [0] * len(admitted)
        rows = int(np.sum(n))
        if rows > self.max_rows:
            raise ValueError(f"iteration {t}: {rows} rows exceed the {self.max_rows}-row buffers")
        q_indptr = np.zeros(len(items) + 1, np.int32)
        q_indptr[1:] = np.cumsum(n)
        kv_len = np.asarray([s.L for s in items], np.int32)
        page_indptr = np.zeros(len(items) + 1, np.int32)
        page_indptr[1:] = np.cumsum([len(s.pages) for s in items])
        page_ids = np.concatenate([np.asarray(s.pages, np.int32) for s in items])
        t0 = time.perf_counter()
        p = attn.plan(q_indptr=q_indptr, q_offset=np.asarray(o, np.int32), kv_len=kv_len,
                      page_indptr=page_indptr, page_ids=page_ids, num_q_heads=self.hq,
                      num_kv_heads=self.hkv, head_dim=self.d, num_pool_pages=self.pool.num_pages,
                      sm_scale=self.sm_scale, device=self.dev)
        plan_ms = (time.perf_counter() - t0) * 1e3
        if self.dev is None:
            timed = capture = False
        else:
            self._nd = nd
            self._desc = (q_indptr, np.asarray(o, np.int32), kv_len, page_indptr)
            self._left = None
            self._run(p, page_ids, rows, timed, capture, items)
        rec = Iteration(t=t, decodes=len(decodes), prefills=len(admitted),
                        prefill_tokens=int(sum(s.L for s in admitted)), waiting_after=len(self.waiting),
                        deficit=self.deficit, plan_ms=plan_ms, events=self._ev if timed else None,
                        launch_events=self._lev if timed else None,
                        queue_waits=[t - s.queued_at for s in admitted])
        rec.captured = self._snap if capture else None
        rec.batch = [(s.req.rid, "decode" if k < nd else "prefill") for k, s in enumerate(items)]
        if self.dev is not None and self.sampling is not None:
            rec.left = self._left if self._left is not None else []
        self._advance(t, decodes, admitted, rec.left)
        return rec

    def _resize(self, s: _State, length: int) -> None:
        """A request's length in the block table, from the next batch on."""
        if self.dev is not None:
            self._changes[-1].append((self._rows[id(s)], length))

    def _batch_tables(self, items, rows: int, pages: int) -> tables.Tables:
        """The block table after this iteration's requests, and what the batch's
        calls read of it: the host sends lengths and offsets."""
        for change in self._changes:  # (pages go back and are taken in the host's order)
            if change:
                at, length = zip(*change)
                self._lengths[list(at)] = length
                self._short.append(tables.resize(self.table, self.held, torch.from_numpy(self._lengths.copy()).to(self.dev, non_blocking=True),
                                                 self.free_pages, self.num_free))
        self._changes = [[]]
        q_indptr, q_offset, kv_len, _ = self._desc
        n = len(items)
        sent = torch.from_numpy(np.concatenate([np.asarray([self._rows[id(s)] for s in items], np.int32), kv_len, q_offset, q_indptr])).to(self.dev, non_blocking=True)
        return tables.build(self.table, sent[:n], sent[n:2 * n], sent[3 * n:], sent[2 * n:3 * n], rows=rows, pages=pages)

    def _positions(self) -> np.ndarray:
        """Position of every row of the batch."""
        q_indptr, q_offset, _, _ = self._desc
        return np.arange(q_indptr[-1], dtype=np.int32) + np.repeat(q_offset - q_indptr[:-1], q_indptr[1:] - q_indptr[:-1])

    def _sample(self, b: tables.Tables, items) -> None:
        """A token for every row of the decodes' blocks, and the rows that keep
        theirs; the responses of fresh prefills are masked first."""
        q_indptr = self._desc[0]
        for k, s in enumerate(items[self._nd:], self._nd):
            if s.fresh:
                self.ids[b.slots[int(q_indptr[k]):int(q_indptr[k + 1])][s.req.prompt:]] = self.mask_id
                s.fresh = False
        rows = BLOCK * self._nd
        if rows == 0:
            return
        if self.logits.shape[0] < rows:  # as a language model's: a broad bulk, and in each row one token that stands out
            self.logits = (2.2 * torch.randn((rows, self.mask_id + 1), generator=self._gen, device=self.dev)).to(torch.bfloat16)
            high = 10.0 + 15.0 * torch.rand((rows, 1), generator=self._gen, device=self.dev)
            self.logits.scatter_(1, torch.randint(0, self.mask_id, (rows, 1), generator=self._gen, device=self.dev), high.to(torch.bfloat16))
        u = torch.rand((rows,), generator=self._gen, device=self.dev)
        tokens, confidence = sample.tokens(self.logits[:rows], u, forbid=self.mask_id, **self.sampling)
        out, left = sample.unmask(tokens, confidence, self.ids, self._indptr(self._nd), mask_id=self.mask_id, count=self.count, threshold=self.threshold,
                                  slots=b.slots[:rows])
        self.sampled = (tokens, confidence, out)
        self._left = self._told(left)  # (the host waits here: the blocks that are done leave the next batch)

    def _told(self, left: torch.Tensor) -> List[int]:
        """A tensor's values on the host, and with them whether the device's free pages were as many as the host's."""
        told = torch.cat([left, *self._short]).tolist() if self._short else left.tolist()
        n = left.numel()
        self._short = []
        if any(told[n:]):
            raise RuntimeError("the block table found too few free pages: it does not follow the host's pool any more")
        return told[:n]

    def _indptr(self, blocks: int) -> torch.Tensor:
        return torch.arange(0, BLOCK * blocks + 1, BLOCK, dtype=torch.int32, device=self.dev)

    def _run(self, p, page_ids, rows, timed, capture, items):
        b = None
        if self.sampling is not None or capture:
            b = self._batch_tables(items, rows, len(page_ids))
            pid = b.page_ids
        else:
            pid = torch.from_numpy(page_ids).to(self.dev, non_blocking=True)
            if self._changes[-1]:
                self._changes.append([])
        stream = torch.cuda.current_stream(self.dev)
        snap = None
        nd = self._nd
        q, k_new, v_new = self.q[:rows], self.k_new[:rows], self.v_new[:rows]
        if self.rope is not None:
            positions = b.positions if b is not None else torch.from_numpy(self._positions()).to(self.dev, non_blocking=True)
            q, k_new = rope.rotate(self.rope, q, k_new, positions, q_out=self.q_rot[:rows], k_out=self.k_rot[:rows])
        if capture:
            q_indptr, q_offset, kv_len, page_indptr = self._desc
            snap = dict(q_indptr=q_indptr, q_offset=q_offset, kv_len=kv_len,
                        page_indptr=page_indptr, page_ids=page_ids, sm_scale=self.sm_scale,
                        q=q.clone(), k_new=k_new.clone(), v_new=v_new.clone(), decodes=nd)
            snap["k_pages"], snap["v_pages"] = self._pages(page_ids, pid)
            snap["tables"] = b
        ev = lev = used = None
        if timed:
            ev = (torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True))
            lev = [torch.cuda.Event(enable_timing=True) for _ in range(6)]
            for e in lev:  # torch reads elapsed time only from events it has recorded
                e.record(stream)
            used = p.launches()
            ev[0].record(stream)
        if self.cache is None:
            attn.forward(p, q, k_new, v_new, self.k_cache, self.v_cache, pid, out=self.out[:rows],
                         lse=self.lse[:rows], launch_events=lev)
        else:
            kvq.forward(p, q, k_new, v_new, self.cache, pid, out=self.out[:rows], lse=self.lse[:rows],
                        launch_events=lev)
        if timed:
            ev[1].record(stream)
            lev = [(lev[2 * k], lev[2 * k + 1]) for k in range(3) if used[k]]
        if self.sampling is not None:
            self._sample(b, items)
        if capture:
            snap["out"] = self.out[:rows].clone()
            snap["lse"] = self.lse[:rows].clone()
        self._ev, self._lev, self._snap = ev, lev, snap

    def _advance(self, t, decodes, admitted, left=None):
        # advance: a prefill starts (or resumes at) its block; a decode step
        # may resolve the block, which sends the request back for a re-prefill
        done = []
        for s in admitted:
            s.phase = "decoding"
            s.steps_left = s.req.steps[s.block]
        for k, s in enumerate(decodes):
            s.steps_left = s.steps_left - 1 if left is None else left[k]
            if s.steps_left == 0:
                s.block += 1
                if s.block == len(s.req.steps):
                    s.phase = "done"
                    done.append(s)
                else:
                    s.phase = "waiting"
                    s.queued_at = t + 1
                    self.waiting.append(s)
        for s in reversed(done):  # in the order of the block table: the first one's pages are taken first
            self.pool.give(s.pages)
            s.pages = None
            self._resize(s, 0)
        self.waiting.sort(key=lambda s: (s.req.arrival, s.req.rid))

    def run(self, max_iterations: int, timed: bool = True) -> List[Iteration]:
        log = []
        for t in range(max_iterations):
            if not self.busy():
                break
            rec = self.step(t, timed)
            if rec is not None:
                log.append(rec)
        if self.dev is not None and self._short:
            self._told(self.num_free)
        return log
