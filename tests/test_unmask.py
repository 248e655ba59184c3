"""Unmasking (include/sangam_sample.h, sample.unmask) against its definition on
the host: counts and thresholds, ties, blocks of no row to thousands, ids in
place, apart and behind slots, refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2607_04206_amd import _lib, sample

MASK = 99999


def definition(tokens, conf, ids, indptr, mask_id, counts, thresholds):
    out, left = ids.copy(), np.zeros(len(indptr) - 1, np.int64)
    for b in range(len(left)):
        rows = [r for r in range(indptr[b], indptr[b + 1]) if ids[r] == mask_id and tokens[r] >= 0 and tokens[r] != mask_id]
        rank = sorted(rows, key=lambda r: (-(conf[r] if conf[r] == conf[r] else -math.inf), conf[r] != conf[r], r))
        for r in set(rank[:max(0, counts[b])]) | {r for r in rows if conf[r] >= thresholds[b]}:
            out[r] = tokens[r]
        left[b] = (out[indptr[b]:indptr[b + 1]] == mask_id).sum()
    return out, left


def case(sizes, seed, how="uniform", masked=0.7):
    rng = np.random.default_rng(seed)
    indptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n = int(indptr[-1])
    conf = rng.random(n).astype(np.float32)
    if how == "ties":
        conf = np.round(conf * 4).astype(np.float32) / 4
    elif how == "negative":  # entropies
        conf = -10 * conf
    elif how == "odd":
        conf = rng.choice(np.array([0.0, -0.0, math.nan, -math.nan, math.inf, -math.inf, 1.0, 1e-45, -1e-45, 0.5, -3.0], np.float32), n)
    ids = np.where(rng.random(n) < masked, MASK, rng.integers(0, 5000, n)).astype(np.int32)
    tokens = rng.integers(0, 5000, n).astype(np.int32)
    tokens[rng.random(n) < 0.05] = -1
    tokens[rng.random(n) < 0.05] = MASK
    return indptr, tokens, conf, ids


@pytest.fixture
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    return torch.device("cuda:0")


def put(dev, *arrays):
    return [torch.from_numpy(np.ascontiguousarray(x)).to(dev) for x in arrays]


SIZES = {"one": [1], "block": [32], "wave": [64, 65, 63, 0, 1, 128], "many": [32] * 301, "ragged": [0, 5, 0, 0, 100, 1, 31, 700, 64, 2], "limit": [1024, 1025, 3],
         "large": [5000, 32, 2049, 0, 1030], "held": [4096, 4097, 0, 2048, 1025, 1, 4095, 257], "spread": [1100, 1536, 700, 1, 0] * 5}


@pytest.mark.gpu
@pytest.mark.parametrize("count,threshold", [(1, math.inf), (0, 0.9), (4, 0.5), (10 ** 9, math.inf), (0, math.inf), (40, 2.0), (2, -math.inf), (900, math.inf)])
@pytest.mark.parametrize("how", ["uniform", "ties", "negative", "odd"])
@pytest.mark.parametrize("sizes", list(SIZES))
def test_blocks(dev, sizes, how, count, threshold):
    for masked in (0.7, 1.0, 0.0):
        indptr, tokens, conf, ids = case(SIZES[sizes], 3, how, masked)
        t = put(dev, tokens, conf, ids, indptr)
        out, left = sample.unmask(*t, mask_id=MASK, count=count, threshold=threshold)
        blocks = len(indptr) - 1
        want, remain = definition(tokens, conf, ids, indptr, MASK, [count] * blocks, [np.float32(threshold)] * blocks)
        assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(left.cpu().numpy(), remain)
        assert np.array_equal(t[2].cpu().numpy(), ids)  # apart
        sample.unmask(*t, mask_id=MASK, count=count, threshold=threshold, out=t[2])
        assert np.array_equal(t[2].cpu().numpy(), want)  # in place


@pytest.mark.gpu
def test_parameters_of_blocks(dev):
    rng = np.random.default_rng(1)
    sizes = rng.integers(0, 90, 57)
    indptr, tokens, conf, ids = case(sizes, 8, "ties")
    counts = rng.integers(-2, 12, 57).astype(np.int32)
    thresholds = rng.choice(np.array([0.25, 0.5, 1.0, math.inf, math.nan, -math.inf], np.float32), 57)
    c, th = put(dev, counts, thresholds)
    out, left = sample.unmask(*put(dev, tokens, conf, ids, indptr), mask_id=MASK, count=c, threshold=th)
    want, remain = definition(tokens, conf, ids, indptr, MASK, counts, thresholds)
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(left.cpu().numpy(), remain)


@pytest.mark.gpu
@pytest.mark.parametrize("mask_id", [MASK, -1])
def test_slots(dev, mask_id):
    """ids in the pool that slots address; rows without a slot, in blocks and behind them."""
    rng = np.random.default_rng(2)
    indptr, tokens, conf, ids = case([32, 0, 70, 1100, 5], 4)
    ids[ids == MASK] = mask_id
    tokens[tokens == MASK] = 17
    rows, pool = len(ids) + 11, 4000  # eleven rows of padding
    slots = np.full(rows, -1, np.int64)
    slots[:len(ids)] = rng.permutation(pool)[:len(ids)]
    gone = np.concatenate([[3, 40, 500], np.arange(len(ids), rows)])
    slots[gone] = rng.choice(np.array([-1, pool, 2 ** 40, -2 ** 40]), len(gone))
    tokens, conf = np.concatenate([tokens, np.zeros(11, np.int32)]), np.concatenate([conf, np.ones(11, np.float32)])
    ids = np.concatenate([ids, np.zeros(11, np.int32)])
    there = (slots >= 0) & (slots < pool)
    held = rng.integers(0, 5000, pool).astype(np.int32)
    held[slots[there]] = ids[there]
    t = put(dev, tokens, conf, held, indptr)
    out, left = sample.unmask(*t, mask_id=mask_id, count=3, threshold=0.8, slots=put(dev, slots)[0])
    hidden = np.where(there, ids, 123456)  # (not the mask)
    want, remain = definition(tokens, conf, hidden, indptr, mask_id, [3] * 5, [np.float32(0.8)] * 5)
    assert np.array_equal(out.cpu().numpy(), np.where(there, want, -1)) and np.array_equal(left.cpu().numpy(), remain)
    after = held.copy()
    after[slots[there]] = want[there]
    assert np.array_equal(t[2].cpu().numpy(), after)


@pytest.mark.gpu
def test_rows_outside_blocks_and_bad_offsets(dev):
    indptr, tokens, conf, ids = case([8, 8, 8], 5, masked=1.0)
    t = put(dev, tokens, conf, ids)
    some = torch.tensor([4, 12, 20], dtype=torch.int32, device=dev)
    out, left = sample.unmask(*t, some, mask_id=MASK, count=100)
    want, remain = definition(tokens, conf, ids, [4, 12, 20], MASK, [100] * 2, [math.inf] * 2)
    assert np.array_equal(out.cpu().numpy(), want) and np.array_equal(left.cpu().numpy(), remain)
    # offsets behind the rows or before the first lead nowhere
    wild = torch.tensor([-50, 2 ** 30, 3, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    out, left = sample.unmask(*t, wild, mask_id=MASK, count=1)
    torch.cuda.synchronize()
    assert out.shape == (24,) and left.shape == (3,)
    out, left = sample.unmask(*t, torch.zeros(1, dtype=torch.int32, device=dev), mask_id=MASK)
    assert np.array_equal(out.cpu().numpy(), ids) and left.numel() == 0
    none = [x[:0] for x in t]
    out, left = sample.unmask(*none, torch.zeros(4, dtype=torch.int32, device=dev), mask_id=MASK, left=torch.full((3,), 7, dtype=torch.int32, device=dev))
    assert out.numel() == 0 and left.tolist() == [0, 0, 0]


def test_definition():
    ids = np.array([MASK, 5, MASK, MASK, MASK], np.int32)
    out, left = definition(np.array([1, 2, 3, -1, 4], np.int32), np.array([0.2, 0.9, 0.2, 1.0, 0.1], np.float32), ids, [0, 5], MASK, [1], [2.0])
    assert out.tolist() == [1, 5, MASK, MASK, MASK] and left.tolist() == [3]


def c_desc(**kw):
    d = _lib.UnmaskDesc(4096, 4096, 4096, None, 4096, None, None, 8, 8, 1, 7, 1, 0.9)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("status,kw", [
    (-1, dict(rows=-1)), (-1, dict(rows=2 ** 31)), (-1, dict(num_blocks=-1)), (-1, dict(num_ids=-1)), (-1, dict(num_ids=7)), (-1, dict(count=-1)),
    (-1, dict(threshold=math.nan)), (-1, dict(row_indptr=None)), (-1, dict(tokens=None)), (-1, dict(confidence=None)), (-1, dict(ids=None)),
    (-6, dict(tokens=4097)), (-6, dict(ids=4098)), (-6, dict(slots=4100)), (-6, dict(counts=4097)), (-6, dict(thresholds=4097)), (-6, dict(row_indptr=4099))])
def test_c_refusals(status, kw):
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc(**kw)), 4096, 4096, None) == status


def test_c_outputs_refused():
    assert _lib.lib.sangam_sample_unmask(None, 4096, 4096, None) == -1
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc()), None, 4096, None) == -1
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc()), 4097, 4096, None) == -6
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc()), 4096, 4098, None) == -6
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc(rows=0, num_ids=0, num_blocks=0)), None, None, None) == 0


@pytest.mark.gpu
def test_python_refusals(dev):
    n = 8
    t = dict(tokens=torch.zeros(n, dtype=torch.int32, device=dev), confidence=torch.zeros(n, device=dev), ids=torch.zeros(n, dtype=torch.int32, device=dev),
             row_indptr=torch.tensor([0, n], dtype=torch.int32, device=dev), mask_id=7)
    for error, kw in [(TypeError, dict(tokens=t["confidence"])), (ValueError, dict(confidence=t["confidence"][:3])), (ValueError, dict(ids=t["ids"][:3])),
                      (TypeError, dict(ids=t["ids"].long())), (ValueError, dict(row_indptr=t["row_indptr"][:0])), (ValueError, dict(count=-1)),
                      (ValueError, dict(threshold=math.nan)), (ValueError, dict(count=t["ids"])), (TypeError, dict(threshold=t["ids"][:1])),
                      (TypeError, dict(slots=t["ids"])), (ValueError, dict(slots=t["ids"].long()[:3])), (ValueError, dict(out=t["ids"][:3])),
                      (ValueError, dict(left=t["ids"])), (ValueError, dict(ids=t["ids"].cpu()))]:
        with pytest.raises(error):
            sample.unmask(**{**t, **kw})


@pytest.mark.gpu
@pytest.mark.parametrize("mask_id", [2 ** 31, 2 ** 32 + 7, -2 ** 31 - 1, -2 ** 40])
def test_mask_past_32_bits_is_refused(dev, mask_id):
    """A mask that no id can be is not taken for the one that its last 32 bits are."""
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    with pytest.raises(ValueError, match="mask_id"):
        sample.unmask(ints(1, 2), torch.ones(2, device=dev), ints(7, 7), ints(0, 2), mask_id=mask_id)
    for edge in (2 ** 31 - 1, -2 ** 31):
        out, left = sample.unmask(ints(1, 2), torch.ones(2, device=dev), ints(edge, 7), ints(0, 2), mask_id=edge, count=0)
        assert out.tolist() == [edge, 7] and left.tolist() == [1]


@pytest.mark.gpu
def test_blocks_past_32_bits_are_refused(dev):
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    with pytest.raises(ValueError, match="row_indptr"):
        sample.unmask(ints(1, 2), torch.ones(2, device=dev), ints(7, 7), torch.empty(2 ** 32 + 2, dtype=torch.int32, device=dev), mask_id=7,
                      left=ints(0))


@pytest.mark.parametrize("rows", [0, 8, 2 ** 31 - 1])
def test_more_blocks_than_a_launch_takes(rows):
    """The header's limit, whatever the rows (a call without rows has a launch as well, for left)."""
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc(rows=rows, num_ids=rows, num_blocks=4 * (2 ** 24 - 1) + 1)), 4096, 4096, None) == -1
    assert b"num_blocks" in _lib.lib.sangam_last_error()
    assert _lib.lib.sangam_sample_unmask(ctypes.byref(c_desc(rows=0, num_ids=0, num_blocks=4 * (2 ** 24 - 1) + 1)), None, None, None) == -1


@pytest.mark.gpu
def test_as_many_blocks_as_a_launch_takes(dev):
    blocks, n = 4 * (2 ** 24 - 1), 8
    indptr = torch.zeros(blocks + 1, dtype=torch.int32, device=dev)
    indptr[blocks // 2:] = 3
    indptr[-1] = n
    ids = torch.full((n,), MASK, dtype=torch.int32, device=dev)
    conf = torch.tensor([0.1, 0.3, 0.2, 0.5, 0.4, 0.7, 0.6, 0.0], device=dev)
    out, left = sample.unmask(torch.arange(n, dtype=torch.int32, device=dev), conf, ids, indptr, mask_id=MASK, count=1)
    assert out.tolist() == [MASK, 1, MASK, MASK, MASK, 5, MASK, MASK]
    at = left.nonzero()[:, 0]
    assert at.tolist() == [blocks // 2 - 1, blocks - 1] and left[at].tolist() == [2, 4]


@pytest.mark.gpu
@pytest.mark.parametrize("slotted", [False, True])
@pytest.mark.parametrize("blocks,rows", [(3, 24), (1, 700), (40, 9000), (500, 6000)])
def test_wrong_contents(dev, blocks, rows, slotted):
    """Whatever offsets, slots, counts and thresholds hold: nothing around the outputs is written, and a row's id afterwards is its
    own, its token or, without a slot, -1."""
    rng = np.random.default_rng(blocks)
    kept, pool = -987654, 2 * rows
    for trial in range(6):
        indptr = np.where(rng.random(blocks + 1) < 0.6, rng.integers(-20, rows + 20, blocks + 1), rng.choice([-2 ** 31, 2 ** 31 - 1, -1, 0, 2 ** 30], blocks + 1))
        if trial >= 3:
            indptr = np.sort(indptr)
        _, tokens, conf, ids = case([rows], trial, "odd")
        counts, thresholds = rng.choice(np.array([-2 ** 31, -1, 0, 3, 2 ** 31 - 1]), blocks), rng.choice(np.array([math.nan, math.inf, -math.inf, 0.5]), blocks)
        if slotted:
            slots = rng.permutation(pool)[:rows]
            wild = rng.random(rows) < 0.2
            slots[wild] = rng.choice(np.array([-1, pool, 2 ** 62, -2 ** 63, 2 ** 40]), int(wild.sum()))
            there = (slots >= 0) & (slots < pool)
            held = rng.integers(5000, 6000, pool)
            held[slots[there]] = ids[there]
        else:
            there, held = np.ones(rows, bool), ids
        def guarded(n, x=None):  # noqa: E306
            t = torch.full((n + 64,), kept, dtype=torch.int32, device=dev)
            if x is not None:
                t[32:32 + n] = torch.from_numpy(x.astype(np.int32)).to(dev)
            return t
        around = [guarded(len(held), held), guarded(rows), guarded(blocks)]
        pool_ids, out, left = (t[32:-32] for t in around)
        sample.unmask(*put(dev, tokens, conf), pool_ids, *put(dev, indptr.astype(np.int32)), mask_id=MASK, count=put(dev, counts.astype(np.int32))[0],
                      threshold=put(dev, thresholds.astype(np.float32))[0], slots=put(dev, slots)[0] if slotted else None, out=out, left=left)
        torch.cuda.synchronize()
        assert all((t[:32] == kept).all() and (t[-32:] == kept).all() for t in around)
        got = out.cpu().numpy()
        assert ((got == ids) | ((ids == MASK) & (tokens >= 0) & (got == tokens)))[there].all() and (got[~there] == -1).all()
        after = pool_ids.cpu().numpy()
        if slotted:
            assert ((after[slots[there]] == ids[there]) | ((ids == MASK) & (after[np.where(there, slots, 0)] == tokens))[there]).all()
            rest = np.ones(pool, bool)
            rest[slots[there]] = False
            assert np.array_equal(after[rest], held[rest])
        else:
            assert np.array_equal(after, ids)
        assert (left != kept).all()
