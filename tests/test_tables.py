"""Page tables (include/sangam_tables.h, paper_2607_04206_amd/tables.py) against
host lists: requests that grow and shrink over a stack of free pages, and the
page list, positions, slots and items of a batch. Whole numbers: all equal."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2607_04206_amd import _lib, tables
from paper_2607_04206_amd.serve import PagePool

PAGE = 16


@pytest.fixture
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    return torch.device("cuda:0")


def put(dev, x, dtype=torch.int32):
    return torch.tensor(np.asarray(x).astype(np.int64), dtype=dtype, device=dev)


class Host:
    """The same tables as lists."""

    def __init__(self, requests, max_pages, pool, rng):
        self.lists, self.max_pages = [[] for _ in range(requests)], max_pages
        self.free = [int(p) for p in rng.permutation(pool)]

    def resize(self, lengths):
        need = [-(-max(0, int(n)) // PAGE) for n in lengths]
        back = []
        for pages, n in zip(self.lists, need):
            back += pages[n:]
            del pages[n:]
        self.free += reversed(back)
        short, ended = 0, False
        for pages, n in zip(self.lists, need):
            more = n - len(pages)
            if n > self.max_pages:
                short += 1
            elif more > 0:
                ended = ended or more > len(self.free)
                if ended:
                    short += 1
                else:
                    pages += [self.free.pop() for _ in range(more)]
        return short


def device_tables(dev, host, pool, extra=0):
    requests = len(host.lists)
    buffer = torch.full((requests, host.max_pages + extra), -5, dtype=torch.int32, device=dev)
    table = buffer[:, :host.max_pages]
    table.fill_(-1)
    free = torch.full((pool,), -9, dtype=torch.int32, device=dev)
    free[:len(host.free)] = put(dev, host.free)
    return buffer, table, put(dev, np.zeros(requests)), free, put(dev, [len(host.free)])


def same(host, buffer, table, held, free, num_free):
    assert held.tolist() == [len(p) for p in host.lists] and num_free.tolist() == [len(host.free)]
    assert free[:len(host.free)].tolist() == host.free
    rows = table.tolist()
    for pages, row in zip(host.lists, rows):
        assert row == pages + [-1] * (host.max_pages - len(pages))
    if buffer.shape[1] > table.shape[1]:
        assert (buffer[:, table.shape[1]:] == -5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("requests,max_pages,pool,extra", [(1, 1, 1, 0), (1, 300, 200, 0), (5, 7, 20, 3), (64, 40, 1000, 0), (1024, 12, 5000, 1), (1025, 9, 3000, 0),
                                                           (3000, 20, 20000, 5), (7, 1000, 3000, 0)])
def test_resize(dev, requests, max_pages, pool, extra):
    """Steps of growing, shrinking, coming, going, and too few pages."""
    rng = np.random.default_rng(requests)
    host = Host(requests, max_pages, pool, rng)
    t = device_tables(dev, host, pool, extra)
    lengths = np.zeros(requests, np.int64)
    for step in range(12):
        change = rng.random(requests)
        share = rng.choice([0.02, 0.3, 1.0])
        lengths = np.where(change < share, rng.integers(0, max_pages * PAGE + 1, requests) * (rng.random(requests) < 0.6), lengths)
        lengths = np.where(rng.random(requests) < 0.01, rng.choice([-3, max_pages * PAGE + 1, 2 ** 31 - 1]), lengths)
        short = tables.resize(t[1], t[2], put(dev, lengths), t[3], t[4])
        assert short.tolist() == [host.resize(lengths)], f"step {step}"
        same(host, *t)


@pytest.mark.gpu
def test_resize_follows_the_pool(dev):
    """The order of pages is that of the host's pool: what one request gave back last it takes first."""
    pool = PagePool(50)
    order = pool._free[:]
    free, num_free, held = put(dev, order), put(dev, [50]), put(dev, [0, 0, 0])
    table = torch.full((3, 20), -1, dtype=torch.int32, device=dev)
    a, b = pool.take(5), pool.take(20)
    tables.resize(table, held, put(dev, [80, 320, 0]), free, num_free)
    assert table[0, :5].tolist() == a and table[1].tolist() == b
    pool.give(a)
    c = pool.take(7)
    tables.resize(table, held, put(dev, [0, 305, 100]), free, num_free)
    assert table[2, :7].tolist() == c and table[0].tolist() == [-1] * 20 and num_free.tolist() == [pool.free]


@pytest.mark.gpu
def test_resize_of_wrong_contents(dev):
    """Counts beyond their arrays lead nowhere."""
    table = torch.arange(40, dtype=torch.int32, device=dev).view(4, 10)
    guard = torch.full((64,), -77, dtype=torch.int32, device=dev)
    free = guard[8:28]
    free.copy_(torch.arange(100, 120))
    held, num_free = put(dev, [2 ** 31 - 1, -4, 10, 3]), put(dev, [2 ** 31 - 1])
    tables.resize(table, held, put(dev, [0, 160, 0, 33]), free, num_free)
    torch.cuda.synchronize()
    assert (guard[:8] == -77).all() and (guard[28:] == -77).all()
    assert held.tolist()[0] == 0 and 0 <= int(num_free) <= 20
    tables.resize(table, held, put(dev, [160] * 4), free, put(dev, [-5]))
    torch.cuda.synchronize()


def batch(rng, requests, items, longest, padding=0, listed=False):
    host = dict(request=rng.integers(0, requests, items), kv_len=rng.integers(0, longest + 1, items))
    n = np.where(rng.random(items) < 0.2, host["kv_len"], np.minimum(rng.integers(0, 40, items), host["kv_len"]))
    host["q_indptr"] = np.concatenate([[0], np.cumsum(n)])
    host["q_offset"] = (rng.random(items) * (host["kv_len"] - n + 1)).astype(np.int64)
    host["rows"] = int(n.sum()) + padding
    host["pages"] = int((-(-host["kv_len"] // PAGE)).sum()) + padding
    host["q_pos"] = rng.integers(-3, longest + 20, host["rows"]) if listed else None
    return host


def expected(table, b):
    page_indptr, ids, positions, slots, items = [0], [], [], [], []
    for i, (r, n) in enumerate(zip(b["request"], b["kv_len"])):
        row = table[r] if 0 <= r < len(table) else [-1] * table.shape[1]
        pages = min(-(-int(n) // PAGE), table.shape[1])
        ids += [int(p) for p in row[:pages]]
        page_indptr.append(page_indptr[-1] + pages)
        for k in range(b["q_indptr"][i], b["q_indptr"][i + 1]):
            pos = int(b["q_offset"][i] + k - b["q_indptr"][i]) if b["q_pos"] is None else int(b["q_pos"][k])
            there = 0 <= pos < n and pos // PAGE < table.shape[1] and row[pos // PAGE] >= 0
            positions.append(pos)
            slots.append(int(row[pos // PAGE]) * PAGE + pos % PAGE if there else -1)
            items.append(i)
    more = b["rows"] - len(positions)
    return (page_indptr, (ids + [-1] * b["pages"])[:b["pages"]], positions + [0] * more, slots + [-1] * more, items + [-1] * more)


def built(dev, table, b, **kw):
    got = tables.build(table, None if b["request"] is None else put(dev, b["request"]), put(dev, b["kv_len"]), put(dev, b["q_indptr"]), put(dev, b["q_offset"]),
                       rows=b["rows"], pages=b["pages"], q_pos=None if b["q_pos"] is None else put(dev, b["q_pos"]), **kw)
    return [x.tolist() for x in (got.page_indptr, got.page_ids, got.positions, got.slots, got.items)]


@pytest.mark.gpu
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("requests,items,longest,padding", [(1, 1, 1, 0), (1, 1, 16, 3), (3, 5, 17, 0), (9, 64, 500, 40), (40, 255, 100, 0), (40, 257, 333, 1), (300, 1024, 90, 7),
                                                            (300, 1025, 90, 0), (77, 3001, 40, 300)])
def test_build(dev, requests, items, longest, padding, listed):
    rng = np.random.default_rng(items)
    host = rng.integers(0, 1 << 28, (requests, -(-longest // PAGE)))  # slots beyond 32 bits
    host[rng.random(host.shape) < 0.02] = -1
    b = batch(rng, requests, items, longest, padding, listed)
    b["request"][rng.random(items) < 0.03] = rng.choice([-1, requests, 2 ** 31 - 1])
    buffer = torch.full((requests, host.shape[1] + 3), 12345, dtype=torch.int32, device=dev)
    buffer[:, :host.shape[1]] = put(dev, host)
    for table in (buffer[:, :host.shape[1]], buffer[:, :host.shape[1]].contiguous()):
        for got, want in zip(built(dev, table, b), expected(host, b)):
            assert got == want


@pytest.mark.gpu
def test_build_of_short_outputs_and_no_items(dev):
    rng = np.random.default_rng(1)
    host = rng.integers(0, 1000, (6, 10))
    b = batch(rng, 6, 6, 160)
    b["request"] = np.arange(6)
    want = expected(host, b)
    short = dict(b, rows=b["rows"] - 5, pages=b["pages"] - 2, request=None)
    got = built(dev, put(dev, host), short)
    assert got[0] == want[0] and got[1] == want[1][:-2] and all(x == y[:-5] for x, y in zip(got[2:], want[2:]))
    none = dict(request=None, kv_len=[], q_indptr=[0], q_offset=[], rows=4, pages=3, q_pos=None)
    assert built(dev, put(dev, host), none) == [[0], [-1] * 3, [0] * 4, [-1] * 4, [-1] * 4]
    wild = dict(b, q_indptr=rng.integers(-2 ** 31, 2 ** 31, 7), kv_len=rng.integers(-2 ** 31, 2 ** 31, 6), q_offset=rng.integers(-2 ** 31, 2 ** 31, 6), rows=50, pages=40)
    built(dev, put(dev, host), wild)  # leads nowhere
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_streams_and_graphs(dev):
    """A captured iteration: resize, then build, with other lengths before every replay."""
    rng = np.random.default_rng(4)
    requests, pool = 20, 400
    host = Host(requests, 12, pool, rng)
    t = device_tables(dev, host, pool)
    lengths, kv_len = put(dev, np.full(requests, 10)), put(dev, np.full(8, 10))
    request, q_indptr, q_offset = put(dev, np.arange(8)), put(dev, np.arange(9) * 4), put(dev, np.zeros(8))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tables.resize(t[1], t[2], lengths, t[3], t[4], stream=side)
    tables.build(t[1], request, kv_len, q_indptr, q_offset, rows=40, pages=100, stream=side)
    torch.cuda.synchronize()
    host.resize(lengths.tolist())
    same(host, *t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        short = tables.resize(t[1], t[2], lengths, t[3], t[4])
        out = tables.build(t[1], request, kv_len, q_indptr, q_offset, rows=40, pages=100)
    for step in range(5):
        n = rng.integers(0, 190, requests)
        lengths.copy_(put(dev, n))
        kv_len.copy_(put(dev, n[:8]))
        graph.replay()
        torch.cuda.synchronize()
        assert short.tolist() == [host.resize(n)]
        same(host, *t)
        b = dict(request=np.arange(8), kv_len=n[:8], q_indptr=np.arange(9) * 4, q_offset=np.zeros(8, np.int64), rows=40, pages=100, q_pos=None)
        want = expected(t[1].cpu().numpy(), b)
        assert [x.tolist() for x in (out.page_indptr, out.page_ids, out.positions, out.slots, out.items)] == [list(x) for x in want]


@pytest.mark.gpu
@pytest.mark.parametrize("items,rows,pages", [(1, 7, 5), (6, 50, 40), (300, 5000, 3000), (1025, 4000, 999), (3000, 17, 0)])
def test_build_of_wrong_contents(dev, items, rows, pages):
    """Whatever the arrays hold: nothing around the outputs is written, no input changes, and what comes out is of the table."""
    rng = np.random.default_rng(items)
    requests, longest, kept = 9, 12, -987654
    for trial in range(6):
        held = rng.integers(0, 1 << 28, (requests, longest))
        held[rng.random(held.shape) < 0.1] = -1
        buffer = torch.full((requests + 2, longest + 5), 77777777, dtype=torch.int32, device=dev)
        table = buffer[1:-1, 2:longest + 2]
        table.copy_(put(dev, held))
        before = buffer.clone()
        wild = lambda n, lo, hi: put(dev, np.where(rng.random(n) < 0.5, rng.integers(lo, hi, n), rng.choice([-2 ** 31, 2 ** 31 - 1, -1, 0, 2 ** 30], n)))  # noqa: E731
        inputs = dict(request=wild(items, -3, requests + 3), kv_len=wild(items, -50, 16 * longest + 90), q_indptr=wild(items + 1, -20, rows + 20),
                      q_offset=wild(items, -100, 300), q_pos=wild(rows, -20, 16 * longest + 20) if trial % 2 else None)
        if trial >= 3:  # in order
            inputs["q_indptr"] = put(dev, np.sort(inputs["q_indptr"].cpu().numpy()))
        copies = {k: None if v is None else v.clone() for k, v in inputs.items()}
        sizes = dict(page_indptr=items + 1, page_ids=pages, positions=rows, slots=rows, items=rows)
        around = {k: torch.full((n + 32,), kept, dtype=torch.int64 if k == "slots" else torch.int32, device=dev) for k, n in sizes.items()}
        out = tables.Tables(**{k: around[k][16:16 + n] for k, n in sizes.items()})
        tables.build(table, inputs["request"], inputs["kv_len"], inputs["q_indptr"], inputs["q_offset"], rows=rows, pages=pages, q_pos=inputs["q_pos"], out=out)
        torch.cuda.synchronize()
        for k, n in sizes.items():
            assert (around[k][:16] == kept).all() and (around[k][16 + n:] == kept).all(), k
            assert (out.__dict__[k] != kept).all(), k
        assert torch.equal(buffer, before) and all(v is None or torch.equal(v, copies[k]) for k, v in inputs.items())
        entries = set(held.ravel().tolist()) | {-1}
        assert set(out.page_ids.tolist()) <= entries
        slots, positions = out.slots.cpu().numpy(), out.positions.cpu().numpy()
        there = slots >= 0
        assert (slots[~there] == -1).all() and set((slots[there] // PAGE).tolist()) <= entries and (slots[there] % PAGE == positions[there] % PAGE).all()
        assert ((out.items >= -1) & (out.items < items)).all()
        n = inputs["kv_len"].cpu().numpy()
        pages_of = np.minimum(np.where(n > 0, (n.astype(np.int64) + PAGE - 1) // PAGE, 0), longest)
        assert out.page_indptr.tolist() == [0] + np.cumsum(pages_of).tolist()


def test_places_among_many_offsets(tmp_path):
    """The search among the offsets of as many items as a batch may have, and of a few, on the host and without overflow."""
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(os.path.dirname(os.path.abspath(__file__)), "sanitize", "offsets_driver.cpp"), "-o", exe], check=True)
    asked = [(n, x) for n in (1, 2, 7, 1000, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 2) for x in (-1, 0, 4, 5, 2 ** 40)]
    r = subprocess.run([exe], input="".join(f"{n} {x}\n" for n, x in asked), capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    assert [int(v) for v in r.stdout.split()] == [-1 if x < 0 else n - 1 if x < 5 else n for n, x in asked]


# ------------------------------------------------------------------ refusals
def c_table(**kw):
    t = _lib.BlockTable(4096, 8, 4, 8)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


@pytest.mark.parametrize("status,table,args", [
    (-1, dict(requests=-1), {}), (-1, dict(requests=2 ** 30 + 1), {}), (-1, dict(max_pages=-1), {}), (-1, dict(pages=None), {}), (-1, dict(row_stride=7), {}), (-1, dict(row_stride=2 ** 40 + 1), {}),
    (-6, dict(pages=4098), {}), (-1, {}, dict(held=None)), (-1, {}, dict(lengths=None)), (-1, {}, dict(free=None)), (-1, {}, dict(cap=-1)),
    (-1, {}, dict(num_free=None)), (-1, {}, dict(short=None)), (-6, {}, dict(held=4097)), (-6, {}, dict(free=4098)), (-6, {}, dict(short=4097))])
def test_resize_refusals(status, table, args):
    a = dict(dict(held=4096, lengths=4096, free=4096, cap=10, num_free=4096, short=4096), **args)
    assert _lib.lib.sangam_tables_resize(ctypes.byref(c_table(**table)), a["held"], a["lengths"], a["free"], a["cap"], a["num_free"], a["short"], None) == status


@pytest.mark.parametrize("status,b,args", [
    (-1, dict(num_items=-1), {}), (-1, dict(num_items=2 ** 30 + 1), {}), (-1, dict(kv_len=None), {}), (-1, dict(q_indptr=None), {}), (-1, dict(q_offset=None), {}), (-6, dict(request=4097), {}),
    (-6, dict(q_pos=4098), {}), (-6, dict(kv_len=4097), {}), (-1, {}, dict(page_indptr=None)), (-1, {}, dict(pages=-1)), (-1, {}, dict(rows=-1)),
    (-1, {}, dict(rows=2 ** 31)), (-1, {}, dict(pages=2 ** 31)), (-6, {}, dict(slots=4100)), (-6, {}, dict(page_ids=4097)), (-6, {}, dict(items=4097))])
def test_build_refusals(status, b, args):
    batch = _lib.TablesBatch(3, 0, None, 4096, 4096, 4096, None)
    for k, v in b.items():
        setattr(batch, k, v)
    a = dict(dict(page_indptr=4096, page_ids=4096, pages=10, positions=4096, slots=4096, items=4096, rows=10), **args)
    assert _lib.lib.sangam_tables_build(ctypes.byref(c_table()), ctypes.byref(batch), a["page_indptr"], a["page_ids"], a["pages"], a["positions"], a["slots"],
                                        a["items"], a["rows"], None) == status


def test_null_refusals():
    assert _lib.lib.sangam_tables_resize(None, 4096, 4096, 4096, 4, 4096, 4096, None) == -1
    assert _lib.lib.sangam_tables_build(ctypes.byref(c_table()), None, 4096, 4096, 4, 4096, 4096, 4096, 4, None) == -1


@pytest.mark.gpu
def test_python_refusals(dev):
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    good = dict(table=ints(4, 6), held=ints(4), lengths=ints(4), free=ints(30), num_free=ints(1))
    for error, kw in [(TypeError, dict(table=ints(24))), (TypeError, dict(table=ints(4, 6).long())), (ValueError, dict(table=ints(6, 4).t())), (ValueError, dict(held=ints(3))),
                      (TypeError, dict(lengths=ints(4).long())), (ValueError, dict(free=ints(60)[::2])), (ValueError, dict(num_free=ints(2))),
                      (ValueError, dict(short=ints(2))), (ValueError, dict(held=ints(4).cpu())), (ValueError, dict(table=ints(1, 6).expand(4, 6)))]:
        with pytest.raises(error):
            tables.resize(**{**good, **kw})
    good = dict(table=ints(4, 6), request=None, kv_len=ints(3), q_indptr=ints(4), q_offset=ints(3), rows=5, pages=7)
    for error, kw in [(ValueError, dict(request=ints(2))), (ValueError, dict(q_indptr=ints(3))), (ValueError, dict(q_offset=ints(4))), (ValueError, dict(q_pos=ints(4))),
                      (ValueError, dict(rows=-1)), (ValueError, dict(pages=-1)), (TypeError, dict(kv_len=ints(3).float())),
                      (ValueError, dict(out=tables.Tables(ints(4), ints(6), ints(5), ints(5).long(), ints(5)))),
                      (TypeError, dict(out=tables.Tables(ints(4), ints(7), ints(5), ints(5), ints(5))))]:
        with pytest.raises(error):
            tables.build(**{**good, **kw})
    with pytest.raises(ValueError, match="GPU"):
        tables.resize(**{k: v.cpu() for k, v in dict(table=ints(4, 6), held=ints(4), lengths=ints(4), free=ints(30), num_free=ints(1)).items()})


@pytest.mark.gpu
def test_sizes_past_32_bits_are_refused(dev):
    """Sizes that the C call takes in 32 bits are not cut down to them."""
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    many = torch.empty(2 ** 32 + 3, dtype=torch.int32, device=dev)  # 2 + 1 entries, modulo 2^32
    with pytest.raises(ValueError, match="free"):
        tables.resize(ints(2, 3), ints(2), ints(2), many, ints(1))
    for table in (many.view(1, -1), many.view(-1, 1)):
        with pytest.raises(ValueError, match="table"):
            tables.resize(table, ints(table.shape[0] % 2 ** 32), ints(table.shape[0] % 2 ** 32), ints(9), ints(1))
        with pytest.raises(ValueError, match="table"):
            tables.build(table, None, ints(1), ints(2), ints(1), rows=1, pages=1)
    with pytest.raises(ValueError, match="kv_len"):
        tables.build(ints(2, 3), None, many[:-1], many, many[:-1], rows=1, pages=1, out=tables.Tables(many, ints(1), ints(1), ints(1).long(), ints(1)))
