"""The quantised KV cache (include/sangam_kvq.h, paper_2607_04206_amd/kvq.py).

CPU: the oracle of the formats against torch's own e4m3 numbers and against
every code; the refusals of the C entries and of the Python calls.
GPU: import and export byte for byte against the oracle, over every bf16 bit
pattern and every code; the attention call against the fp64 oracle on the
values that the codes stand for, and the pages it leaves, byte for byte.

Bars of the attention: outputs as in test_parity (bf16 operands, softmax weights
rounded to bf16). The LSE is a sum of unrounded weights in fp32: a score errs by
at most (D + 2) 2^-24 sum |q k| scale, which is below 130 * 2^-24 * 16 = 1.3e-4
(sum |q k| scale is 7 on average for normal q and k of 128 dims, 16 is over 12
standard deviations more), and the sum of at most 8192 weights, 512 to a lane
after the exchanges, by 512 * 2^-24 = 3e-5 of itself: 2e-4.
"""
import ctypes
import dataclasses

import numpy as np
import pytest
import torch

import workloads
from oracle import mx, oracle
from paper_2607_04206_amd import _lib, attn, kv, kvq
from tests import test_parity as parity

FMTS = ("e4m3", "e2m1")
LSE_ABS = 2e-4


# ------------------------------------------------------------- oracle (CPU)
def test_oracle_codes_are_torch_s():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = mx.values(np.arange(256, dtype=np.uint8), np.full(8, 127, np.uint8), "e4m3")
    assert np.array_equal(got, want, equal_nan=True)
    assert mx.code_values("e2m1").tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6]


@pytest.mark.parametrize("fmt", FMTS)
def test_oracle_quantises_to_the_nearest(fmt):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 64)) * np.exp(3 * rng.standard_normal((40, 1)))
    x = torch.from_numpy(x).bfloat16().double().numpy()
    x[3], x[4, :32], x[5, 7], x[6, 40] = 0.0, 2.0 ** -130, np.inf, np.nan
    codes, scales = mx.quantise(x, fmt)
    back = mx.values(codes, scales, fmt)
    table = np.concatenate([mx.code_values(fmt), -mx.code_values(fmt)])
    for r in range(len(x)):
        for b in range(2):
            block, got, s = x[r, 32 * b:32 * b + 32], back[r, 32 * b:32 * b + 32], int(scales[r, b])
            if not np.isfinite(block).all():
                assert s == 255 and np.isnan(got).all() and not codes.reshape(len(x), 2, -1)[r, b].any()
                continue
            top = table.max() * 2.0 ** (s - 127)
            assert np.abs(block).max() <= top and (s == 10 or np.abs(block).max() > top / 2)
            grid = table * 2.0 ** (s - 127)
            assert np.array_equal(np.abs(block - got), np.abs(block[:, None] - grid).min(1))
    # values are bf16 numbers, and writing them again gives them again
    fine = np.isfinite(back).all(1)
    mx.to_bf16_exact(back)
    again = mx.values(*mx.quantise(back[fine], fmt), fmt)
    assert np.array_equal(again, back[fine])


def test_oracle_matches_torch_casts():
    x = torch.randn(200, 32, generator=torch.Generator().manual_seed(1)).bfloat16()
    codes, scales = mx.quantise(x.double().numpy(), "e4m3")
    y = x.double().numpy() * 2.0 ** (127 - scales.astype(np.float64))
    want = torch.from_numpy(y).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes, want)


# ----------------------------------------------------------- refusals (CPU)
def _kv_plan(hkv=2, d=64):
    return kv.plan(kv_len=[20], page_indptr=[0, 2], page_ids=[1, 0], num_kv_heads=hkv, head_dim=d, num_pool_pages=2)


def _c_cache(**over):
    c = dict(format=1, reserved=0, pool_pages=2, k=4096, v=4096, k_scale=4096, v_scale=4096)
    c.update(over)
    return _lib.KvqCache(*[c[n] for n, _ in _lib.KvqCache._fields_])


@pytest.mark.parametrize("over,status", [(dict(format=0), -2), (dict(format=3), -2), (dict(pool_pages=1), -5), (dict(k=None), -1),
                                         (dict(v_scale=None), -1), (dict(k_scale=None), -1), (dict(v=4096 + 8), -6), (dict(k_scale=4096 + 4), -6)])
def test_copies_refuse(over, status):
    # fake device addresses: every check fails before any HIP call
    p = _kv_plan()
    c = ctypes.byref(_c_cache(**over))
    assert _lib.lib.sangam_kvq_export(p.host_ptr(), 4096, c, 4096, 4096, None) == status
    assert _lib.lib.sangam_kvq_import(p.host_ptr(), 4096, 4096, 4096, c, None) == status
    assert _lib.lib.sangam_last_error()


def test_copies_refuse_plans_and_buffers():
    p, c = _kv_plan(), ctypes.byref(_c_cache())
    junk = np.zeros(512, np.uint8)
    export, import_ = _lib.lib.sangam_kvq_export, _lib.lib.sangam_kvq_import
    assert export(junk.ctypes.data, 4096, c, 4096, 4096, None) == -8
    assert import_(None, 4096, 4096, 4096, c, None) == -8
    assert export(p.host_ptr(), None, c, 4096, 4096, None) == -1
    assert export(p.host_ptr(), 4096, None, 4096, 4096, None) == -1
    assert export(p.host_ptr(), 4096, c, 4096, None, None) == -1
    assert import_(p.host_ptr(), 4096, 4096 + 2, 4096, c, None) == -6


def _attn_plan():
    wl = workloads.ragged_small(0, hq=4, hkv=2, d=64)
    return attn.plan(q_indptr=wl.q_indptr, q_offset=wl.q_offset, kv_len=wl.kv_len, page_indptr=wl.page_indptr, page_ids=wl.page_ids,
                     num_q_heads=4, num_kv_heads=2, head_dim=64, num_pool_pages=wl.num_pool_pages, sm_scale=wl.sm_scale, force_kv_splits=2)


@pytest.mark.parametrize("over,args,status", [
    (dict(), dict(plan=None), -8), (dict(format=7), {}, -2), (dict(k=None), {}, -1), (dict(k_scale=None), {}, -1), (dict(k_scale=4100), {}, -6),
    (dict(v=4104), {}, -6), (dict(pool_pages=1), {}, -5), (dict(), dict(npid=1), -5), (dict(), dict(q=None), -1), (dict(), dict(out=4104), -6),
    (dict(), dict(wsb=0), -5), (dict(), dict(ws=None), -5), (dict(), dict(lse=4098), -6), (dict(), dict(cache=None), -1)])
def test_forward_refuses(over, args, status):
    p = _attn_plan()
    a = dict(plan=p.host_ptr(), q=4096, out=4096, npid=p.total_pages, ws=4096, wsb=p.workspace_bytes, lse=4096,
             cache=ctypes.byref(_c_cache(**dict(dict(pool_pages=p.num_pool_pages), **over))))
    a.update(args)
    got = _lib.lib.sangam_kvq_forward(a["plan"], 4096, a["q"], 4096, 4096, a["cache"], 4096, a["npid"], a["out"], a["lse"], a["ws"], a["wsb"], None, None)
    assert got == status and _lib.lib.sangam_last_error()


def test_caches_are_checked():
    c = kvq.empty_cache(5, 3, 64, format="e2m1")
    assert (c.format, c.num_pool_pages, c.num_kv_heads, c.head_dim) == ("e2m1", 5, 3, 64)
    assert c.k.shape == (5, 3, 16, 32) and c.k_scale.shape == (5, 3, 16, 2)
    e = kvq.empty_cache(5, 3, 128)
    assert e.format == "e4m3" and e.k.dtype == torch.float8_e4m3fn and e.v.shape == (5, 3, 16, 128)
    for bad in (dict(k=e.k.float()), dict(v=e.v[:4]), dict(k_scale=e.k_scale[..., :2]), dict(v_scale=e.v_scale.to(torch.int32)),
                dict(v=c.v), dict(k_scale=e.k_scale.transpose(0, 1).contiguous().transpose(0, 1)), dict(k=None)):
        with pytest.raises((TypeError, ValueError)):
            kvq.QuantCache(**{**dict(k=e.k, v=e.v, k_scale=e.k_scale, v_scale=e.v_scale), **bad})
    with pytest.raises(ValueError):
        kvq.empty_cache(5, 3, 128, format="e5m2")
    with pytest.raises(ValueError):
        kvq.empty_cache(5, 3, 96)
    with pytest.raises(ValueError, match="device"):
        kvq.kv_export(_kv_plan(), kvq.empty_cache(2, 2, 64))
    with pytest.raises(ValueError, match="device"):
        kvq.kv_import(_kv_plan(), None, None, kvq.empty_cache(2, 2, 64))


# ----------------------------------------------------------------- copies (GPU)
@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    return torch.device("cuda:0")


def _put(a: np.ndarray, dev, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev).view(dtype)


def equal(a: np.ndarray, b: np.ndarray, what: str) -> None:
    bad = np.flatnonzero((a != b).reshape(-1)) if a.shape == b.shape else None
    if bad is None or len(bad):
        pytest.fail(f"{what}: shapes {a.shape} and {b.shape}" if bad is None else
                    f"{what}: {len(bad)} of {a.size} differ, the first at {np.unravel_index(bad[0], a.shape)}: "
                    f"{a.reshape(-1)[bad[0]]}, not {b.reshape(-1)[bad[0]]}", pytrace=False)


def _bytes(t: torch.Tensor) -> np.ndarray:
    return t.view(torch.uint8).cpu().numpy()


def _cache_of(codes, scales, fmt, dev):
    """codes, scales: (k, v) arrays"""
    dtype = kvq.FORMATS[fmt][1]
    return kvq.QuantCache(_put(codes[0], dev, dtype), _put(codes[1], dev, dtype), _put(scales[0], dev, torch.uint8), _put(scales[1], dev, torch.uint8))


def _junk_pool(rng, pages, hkv, d, fmt):
    codes = [rng.integers(0, 256, (pages, hkv, 16, d if fmt == "e4m3" else d // 2), np.uint8) for _ in range(2)]
    scales = [rng.integers(100, 150, (pages, hkv, 16, d // 32), np.uint8) for _ in range(2)]
    if fmt == "e4m3":
        codes = [np.where(c & 0x7F == 0x7F, 0, c).astype(np.uint8) for c in codes]
    return codes, scales


def _place(c, pages):
    """(page, slot) of each packed row."""
    page = np.concatenate([pages[c.page_indptr[i] + np.arange(n) // 16] for i, n in enumerate(c.kv_len)])
    return page, np.concatenate([np.arange(n) % 16 for n in c.kv_len])


def _rows(rng, n, hkv, d, kind):
    if kind == "patterns":  # every bf16 bit pattern, neighbours in one block, then in another order
        total = n * hkv * d
        bits = np.arange(total, dtype=np.int64) % 65536
        k = bits.astype(np.uint16)
        v = ((bits * 40503) % 65536).astype(np.uint16)
        v = np.where(v & 0x7F80 == 0x7F80, 0x3F80, v).astype(np.uint16)  # magnitudes of all sizes in one block, all finite
        return k.reshape(n, hkv, d), v.reshape(n, hkv, d)
    x = rng.standard_normal((2, n, hkv, d)) * np.exp(4 * rng.standard_normal((2, n, hkv, d // 32)).repeat(32, -1))
    x[rng.random(x.shape) < 0.02] = 0.0
    x[:, ::7, :, :32] = 0.0
    return tuple(torch.from_numpy(y).bfloat16().view(torch.int16).numpy().view(np.uint16) for y in x)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hkv,d,lengths,kind", [(2, 64, [1, 15, 16, 17, 33, 300, 2, 64], "normal"), (1, 128, [1], "normal"),
                                                (5, 128, [31, 1, 250, 16], "normal"), (3, 64, [700, 9], "patterns"), (4, 128, [129, 257], "patterns")])
def test_import_and_export(dev, fmt, hkv, d, lengths, kind):
    print(f"[case] kvq copies {fmt} {hkv} heads, D {d}, {lengths} {kind}", flush=True)
    c = workloads.kv_transfer_case("kvq", 5, lengths, hkv=hkv, d=d, spare_pages=1)
    rng = np.random.default_rng(len(lengths) + d)
    k, v = _rows(rng, c.rows, hkv, d, kind)
    codes, scales = _junk_pool(rng, c.num_pool_pages, hkv, d, fmt)
    cache = _cache_of(codes, scales, fmt, dev)
    p = kv.plan(kv_len=c.kv_len, page_indptr=c.page_indptr, page_ids=c.dst_pages, num_kv_heads=hkv, head_dim=d, num_pool_pages=c.num_pool_pages, device=dev)
    packed = [_put(x.view(np.int16), dev, torch.bfloat16) for x in (k, v)]
    kvq.kv_import(p, *packed, cache)
    page, slot = _place(c, c.dst_pages)
    got = kvq.kv_export(p, cache)
    for x, co, sc, have, have_s, back in zip((k, v), codes, scales, (cache.k, cache.v), (cache.k_scale, cache.v_scale), got):
        want, want_s = mx.quantise(mx.from_bf16(x), fmt)
        co[page, :, slot], sc[page, :, slot] = want, want_s
        equal(_bytes(have_s), sc, "scales")
        equal(_bytes(have), co, "codes")  # also: no slot past a length, no page off the list was written
        values = mx.to_bf16_exact(mx.values(want, want_s, fmt))
        gotten = back.view(torch.int16).cpu().numpy().view(np.uint16)
        assert np.array_equal(mx.from_bf16(gotten), mx.from_bf16(values), equal_nan=True)
    if kind == "patterns":
        return  # (blocks next to 2^128 read back with infinities)
    # what was read back, written again, is the same values: a hand-off through bf16 loses nothing
    other = kvq.empty_cache(c.num_pool_pages, hkv, d, format=fmt, device=dev)
    kvq.kv_import(p, *got, other)
    for a, b in zip(kvq.kv_export(p, other), got):
        assert np.array_equal(a.view(torch.int16).cpu().numpy(), b.view(torch.int16).cpu().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
def test_export_reads_every_code(dev, fmt):
    """Every code under every scale byte that a writer makes, and under 255."""
    d, hkv = 128, 1
    scale = np.append(np.arange(10, 248), 255).astype(np.uint8)
    bytes_ = np.arange(256, dtype=np.uint8)
    if fmt == "e4m3":
        bytes_ = bytes_[bytes_ & 0x7F != 0x7F]
        bytes_ = np.append(bytes_, [0, 0])
    per = d if fmt == "e4m3" else d // 2
    rows_each = 256 // per
    n = len(scale) * rows_each
    pages = -(-n // 16)
    codes = np.zeros((pages * 16, per), np.uint8)
    codes[:n] = np.tile(bytes_.reshape(rows_each, per), (len(scale), 1))
    scales = np.full((pages * 16, d // 32), 127, np.uint8)
    scales[:n] = scale.repeat(rows_each)[:, None]
    shape = lambda x: x.reshape(pages, 1, 16, -1)  # noqa: E731
    cache = _cache_of([shape(codes)] * 2, [shape(scales)] * 2, fmt, dev)
    p = kv.plan(kv_len=[n], page_indptr=[0, pages], page_ids=np.arange(pages), num_kv_heads=hkv, head_dim=d, num_pool_pages=pages, device=dev)
    want = mx.from_bf16(mx.to_bf16_exact(mx.values(codes[:n], scales[:n], fmt)))
    for got in kvq.kv_export(p, cache):
        got = got.view(torch.int16).cpu().numpy().view(np.uint16)
        assert np.array_equal(mx.from_bf16(got)[:, 0], want, equal_nan=True)


# -------------------------------------------------------------- attention (GPU)
def quantised(wl, fmt):
    """The workload with its cached rows replaced by what their codes stand for."""
    plain = dataclasses.replace(wl)

    def value_fn(item, kind):
        if kind not in (workloads.KIND_KCTX, workloads.KIND_VCTX):
            return wl.value_fn(item, kind) if wl.value_fn else None
        x = plain.k_ctx(item) if kind == workloads.KIND_KCTX else plain.v_ctx(item)
        return torch.from_numpy(mx.values(*mx.quantise(x.double().numpy(), fmt), fmt)).float()
    return dataclasses.replace(wl, value_fn=value_fn)


def quant_inputs(wl, dev, fmt):
    """Inputs on the device, the cache quantised; and the pool as host arrays.
    Slots without context read as NaN."""
    t = workloads.device_inputs(wl, torch.device("cpu"), fill=float("nan"))
    codes, scales = zip(*(mx.quantise(t[n].double().numpy(), fmt) for n in ("k_cache", "v_cache")))
    cache = _cache_of(codes, scales, fmt, dev)
    return {n: t[n].to(dev) for n in ("q", "k_new", "v_new", "page_ids")}, cache, [c.copy() for c in codes], [s.copy() for s in scales]


def plan_of(wl, dev=None, **kw):
    return attn.plan(q_indptr=wl.q_indptr, q_offset=wl.q_offset, kv_len=wl.kv_len, page_indptr=wl.page_indptr, page_ids=wl.page_ids,
                     num_q_heads=wl.num_q_heads, num_kv_heads=wl.num_kv_heads, head_dim=wl.head_dim, num_pool_pages=wl.num_pool_pages,
                     sm_scale=wl.sm_scale, q_pos=wl.q_pos, device=dev, **kw)


def expected_pool(wl, codes, scales, fmt):
    codes, scales = [c.copy() for c in codes], [s.copy() for s in scales]
    for i in range(wl.num_items):
        pos = wl.positions(i)
        pages = wl.item_pages(i)[pos // 16]
        for x, c, s in zip((wl.k_new(i), wl.v_new(i)), codes, scales):
            c[pages, :, pos % 16], s[pages, :, pos % 16] = mx.quantise(x.double().numpy(), fmt)
    return codes, scales


def check_pool(cache, codes, scales):
    for have, want in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), (*codes, *scales)):
        equal(_bytes(have), want, "pool")


def check_attention(wl, out, lse, **kw):
    ref, ref_lse = oracle.attention_all(wl)
    parity.compare(wl.name, out.float().cpu().numpy(), ref, **kw)
    if lse is not None:
        d = np.abs(lse.cpu().numpy().astype(np.float64) - ref_lse).max()
        assert d <= LSE_ABS, f"lse max |delta| {d:.3e}"


def run_case(wl, dev, fmt, **kw):
    print(f"[case] kvq {fmt} {wl.name} seed={wl.seed} items={wl.num_items} {kw}", flush=True)
    wl = quantised(wl, fmt)
    t, cache, codes, scales = quant_inputs(wl, dev, fmt)
    p = plan_of(wl, dev, **kw)
    out, lse = kvq.forward(p, t["q"], t["k_new"], t["v_new"], cache, t["page_ids"])
    torch.cuda.synchronize()
    check_attention(wl, out, lse)
    check_pool(cache, *expected_pool(wl, codes, scales, fmt))
    return p, t, cache, out, lse, wl


SHAPES = [(4, 4, 64), (8, 2, 64), (18, 2, 64), (10, 2, 64), (28, 4, 128), (32, 32, 128), (8, 4, 128), (11, 1, 128), (9, 3, 128), (1, 1, 64), (16, 1, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_ragged_batches(dev, fmt, hq, hkv, d):
    run_case(workloads.ragged_small(0, hq=hq, hkv=hkv, d=d), dev, fmt)


# decodes of every group size, past the sizes that small batches take heads-across tiles for
@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("group,d,splits", [(g, d, s) for g in range(1, 9) for d, s in ((128, 0), (64, 3))] + [(16, 128, 2), (1, 128, 20)])
def test_decode_tiles(dev, fmt, group, d, splits):
    dec = [(40, 300), (200, 1100), (64, 96), (5, 37), (0, 33), (0, 1), (700, 1500), (64, 128)]
    wl = workloads.make_workload(f"decode_g{group}", 11, hq=2 * group, hkv=2, d=d, decodes=dec, prefills=[])
    p, *_ = run_case(wl, dev, fmt, force_kv_splits=splits, num_cus=8)
    assert p.info.num_decode_tiles > 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d", [(32, 32, 128), (28, 4, 128), (8, 8, 64)])
def test_listed_positions(dev, fmt, hq, hkv, d):
    wl = workloads.token_cache_decodes(3, hq=hq, hkv=hkv, d=d, count=5, median=200)
    run_case(wl, dev, fmt)
    run_case(wl, dev, fmt, force_kv_splits=3)


def listed_decodes(hq, hkv, d, prefills=()):
    """Decodes of listed positions beside block decodes: few and many rows, within a page and far apart, at the ends of the
    context and of pages, across 64-key stages that hold none."""
    rng = np.random.default_rng(hq + d)
    pos = [(np.sort(rng.choice(n, min(32, r), replace=False)), n) for n, r in ((300, 32), (1100, 17), (700, 32), (40, 9), (1500, 2))]
    pos += [([0, 33], 34), ([15, 16, 63, 64, 127, 128, 191], 192), ([5, 900], 901), (np.r_[0:16, 500:516], 600), ([70], 71)]
    return workloads.make_workload("listed", 9, hq=hq, hkv=hkv, d=d, decodes=[(40, 300), (200, 1100)], prefills=list(prefills), pos_decodes=pos)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", range(1, 9))
def test_listed_positions_in_decode_tiles(dev, fmt, group, d):
    """The tiles of every group size, whose staging differs, whole and split."""
    for splits in (0, 3):
        p, *_ = run_case(listed_decodes(2 * group, 2, d), dev, fmt, num_cus=8, force_kv_splits=splits)
        assert p.info.num_decode_tiles > 0 and p.info.num_fused_decode_tiles == 0 and p.info.decode_q_waves == group


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,prefills", [(8, 8, 128, [1300, 1025]), (8, 8, 128, [333]), (8, 8, 64, [400, 77]), (14, 2, 128, [333]), (8, 2, 64, [400])])
def test_listed_positions_beside_prefills(dev, fmt, hq, hkv, d, prefills):
    p, *_ = run_case(listed_decodes(hq, hkv, d, prefills), dev, fmt)
    assert p.launches()[:2] == (True, False)  # with MHA decodes in one launch, groups fused into the prefills' tiles
    assert (p.info.num_decode_tiles > 0) == (hq == hkv) and (p.info.num_fused_decode_tiles > 0) == (hq != hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,decodes,prefills", [
    (8, 8, 128, [(64, 1000)] * 6, [1300, 1025]),   # MHA decodes beside wide prefills in one launch
    (4, 4, 64, [(64, 500)] * 6, [400, 77]),         # the same at head dim 64
    (14, 2, 128, [(64, 700), (3, 450)], [333]),     # decodes fused into the prefills' launch
    (4, 2, 128, [], [1100, 1024]),                  # wide tiles alone
    (4, 2, 128, [(3, 9000)], [65])])                # a context that is always split
def test_mixed_batches(dev, fmt, hq, hkv, d, decodes, prefills):
    run_case(workloads.make_workload("mixed", 2, hq=hq, hkv=hkv, d=d, decodes=decodes, prefills=prefills), dev, fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,items", [
    (4, 2, 128, [(100, 700, 200), (0, 300, 64), (17, 50, 33), (0, 1, 1), (8, 9, 1)]),
    (4, 4, 64, [(100, 700, 200), (0, 300, 64), (17, 50, 33), (250, 350, 100)]),
    (2, 2, 128, [(500, 2000, 1030)]),  # wide tiles
    (2, 1, 128, [(1500, 4000, 1024)])])
def test_long_blocks_over_cached_context(dev, fmt, hq, hkv, d, items):
    """Blocks of (offset, length, rows), mostly of more than 32 rows."""
    run_case(workloads.make_workload("blocks", 4, hq=hq, hkv=hkv, d=d, decodes=items, prefills=[]), dev, fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
def test_streams_graphs_and_events(dev, fmt):
    """The same bits on another stream, with events, without an LSE, from a
    caller's workspace, and from a graph replayed between eager calls."""
    wl = workloads.make_workload("streams", 5, hq=8, hkv=8, d=128, decodes=[(64, 900), (200, 1500)], prefills=[130])
    p, t, cache, out0, lse0, wl = run_case(wl, dev, fmt, force_kv_splits=3)
    assert p.workspace_bytes > 0
    args = (p, t["q"], t["k_new"], t["v_new"], cache, t["page_ids"])
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    s = torch.cuda.Stream(dev)
    out, lse = kvq.forward(*args, stream=s)
    s.synchronize()
    assert same(out, out0) and torch.equal(lse, lse0)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(6)]
    for e in ev:
        e.record()
    out, lse = kvq.forward(*args, want_lse=False, launch_events=ev)
    torch.cuda.synchronize()
    assert lse is None and same(out, out0) and ev[0].elapsed_time(ev[1]) > 0
    ws = torch.empty(p.workspace_bytes, dtype=torch.uint8, device=dev)
    out, lse = torch.empty_like(out0), torch.empty_like(lse0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        kvq.forward(*args, out=out, lse=lse, workspace=ws)
    s.synchronize()
    with torch.cuda.graph(g, stream=s):
        kvq.forward(*args, out=out, lse=lse, workspace=ws)
    for _ in range(4):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert same(out, out0) and torch.equal(lse, lse0)
        again, _ = kvq.forward(*args)
        assert same(again, out0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,prefills,kw", [
    *((2 * g, 2, d, [], dict(num_cus=8)) for g in range(1, 9) for d in (64, 128)),  # decode tiles of every group
    (4, 4, 128, [], dict(force_kv_splits=3)), (14, 2, 128, [], dict(force_kv_splits=3, num_cus=8)),
    (8, 8, 128, [1300], {}), (4, 4, 64, [400], {}),  # MHA decodes beside prefills
    (14, 2, 128, [333], {}), (4, 2, 128, [1100], {})])
def test_equal_rows_of_v(dev, fmt, hq, hkv, d, prefills, kw):
    """Where all rows of V are the same, so is every output, whatever the weights: what multiplies V and
    what the sum is divided by are the same numbers. Values that both formats hold, so that cached and
    fresh rows agree, under scores of deviation 8, whose largest weights round far from 1. Products of
    two bf16 numbers are exact and sums of up to 1500 of one sign are off by 1500 * 2^-24 of themselves,
    as is the divisor: 2^-12, below the 2^-9 at which a bf16 number rounds to another."""
    print(f"[case] kvq {fmt} equal rows of V {hq}/{hkv} heads of {d}, prefills {prefills} {kw}", flush=True)
    wl = workloads.make_workload("equal", 8, hq=hq, hkv=hkv, d=d, decodes=[(64, 1000), (3, 450), (0, 33), (600, 1500)], prefills=prefills)
    row = np.random.default_rng(hq + d).choice([0.5, -1.0, 1.5, -2.0, 3.0, 4.0, -6.0], size=(hkv, d))
    assert np.array_equal(mx.values(*mx.quantise(row, fmt), fmt), row)

    def value_fn(item, kind):
        n = {workloads.KIND_VCTX: int(wl.kv_len[item]), workloads.KIND_VNEW: wl.n(item)}.get(kind)
        return None if n is None else torch.from_numpy(row).float().expand(n, hkv, d)
    t, cache, _, _ = quant_inputs(dataclasses.replace(wl, value_fn=value_fn, q_scale=8.0), dev, fmt)
    out, _ = kvq.forward(plan_of(wl, dev, **kw), t["q"], t["k_new"], t["v_new"], cache, t["page_ids"])
    want = np.broadcast_to(row.repeat(hq // hkv, 0), out.shape)
    equal(out.float().cpu().numpy(), want.astype(np.float32), "outputs")


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
def test_values_that_are_no_numbers(dev, fmt):
    """A NaN block of one KV head's cached row makes that head's query heads
    NaN and no others; infinite fresh rows are written as NaN blocks."""
    wl = workloads.make_workload("nan", 6, hq=6, hkv=3, d=128, decodes=[(64, 300)], prefills=[40])
    wl = quantised(wl, fmt)
    t, cache, codes, scales = quant_inputs(wl, dev, fmt)
    p = plan_of(wl, dev)
    clean, _ = kvq.forward(p, t["q"], t["k_new"], t["v_new"], cache, t["page_ids"])
    page = int(wl.item_pages(0)[200 // 16])
    for which in ("k_scale", "v_scale"):
        bad = kvq.QuantCache(cache.k, cache.v, cache.k_scale.clone(), cache.v_scale.clone())
        getattr(bad, which)[page, 1, 200 % 16, 2] = 255
        out, _ = kvq.forward(p, t["q"], t["k_new"], t["v_new"], bad, t["page_ids"])
        nan = torch.isnan(out[:32].float())
        dims = nan[:, 2:4] if which == "k_scale" else nan[:, 2:4, 64:96]  # a block of V is 32 of its dims
        assert dims.all() and nan.sum() == dims.numel()
        rest = ~nan
        assert torch.equal(out[:32][rest], clean[:32][rest]) and torch.equal(out[32:], clean[32:])
    k_new = t["k_new"].clone()
    k_new[3, 2, 5], k_new[4, 0, 100] = float("inf"), float("-inf")  # rows 67 and 68 of the block decode
    kvq.forward(p, t["q"], k_new, t["v_new"], cache, t["page_ids"])
    at = int(wl.item_pages(0)[67 // 16])
    assert cache.k_scale[at, 2, 67 % 16].tolist()[0] == 255 and cache.k_scale[at, 0, 68 % 16].tolist()[3] == 255
    assert int((cache.k_scale[at] == 255).sum()) == 2
    assert not cache.k.view(torch.uint8)[at, 2, 67 % 16, :32 if fmt == "e4m3" else 16].any()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
def test_pages_far_apart(dev, fmt):
    """Pages past 2^32 bytes of the pool: the bits of the same call on a small one."""
    hkv, d = 8, 128
    wl = workloads.make_workload("far", 7, hq=8, hkv=hkv, d=d, decodes=[(64, 500), (0, 40)], prefills=[100])
    wl = quantised(wl, fmt)
    t, small, codes, scales = quant_inputs(wl, dev, fmt)
    pages = 2 ** 32 // (hkv * 16 * small.k.shape[3]) + wl.num_pool_pages + 100
    far = dataclasses.replace(wl, page_ids=(pages - 1 - wl.page_ids).astype(np.int32), num_pool_pages=pages)
    big = kvq.empty_cache(pages, hkv, d, format=fmt, device=dev)
    for a, b in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
        a.view(torch.uint8)[pages - wl.num_pool_pages:] = b.view(torch.uint8).flip(0)
    res = [kvq.forward(plan_of(w, dev), t["q"], t["k_new"], t["v_new"], c, torch.from_numpy(w.page_ids).to(dev)) for w, c in ((wl, small), (far, big))]
    assert torch.equal(res[0][0].view(torch.int16), res[1][0].view(torch.int16)) and torch.equal(res[0][1], res[1][1])
    table = lambda w: kv.plan(kv_len=w.kv_len, page_indptr=w.page_indptr, page_ids=w.page_ids, num_kv_heads=hkv, head_dim=d,  # noqa: E731
                              num_pool_pages=w.num_pool_pages, device=dev)
    rows = [kvq.kv_export(table(w), c) for w, c in ((wl, small), (far, big))]
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(*rows))
    kvq.kv_import(table(far), rows[0][1], rows[0][0], big)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(kvq.kv_export(table(far), big), rows[0][::-1]))
    assert not big.k.view(torch.uint8)[:pages - wl.num_pool_pages].any()


@pytest.mark.gpu
def test_python_refusals(dev):
    wl = workloads.ragged_small(0, hq=4, hkv=2, d=64)
    t = workloads.device_inputs(wl, dev)
    p = plan_of(wl, dev)
    ok = kvq.empty_cache(wl.num_pool_pages, 2, 64, device=dev)
    args = lambda **o: [o.get(n, t[n] if n in t else ok) for n in ("q", "k_new", "v_new", "cache", "page_ids")]  # noqa: E731
    for bad, err in ((dict(q=t["q"].float()), TypeError), (dict(k_new=t["k_new"][:-1]), ValueError), (dict(cache=t["k_cache"]), TypeError),
                     (dict(cache=kvq.empty_cache(wl.num_pool_pages - 1, 2, 64, device=dev)), ValueError),
                     (dict(cache=kvq.empty_cache(wl.num_pool_pages, 1, 64, device=dev)), ValueError),
                     (dict(cache=kvq.empty_cache(wl.num_pool_pages, 2, 128, device=dev)), ValueError),
                     (dict(cache=kvq.empty_cache(wl.num_pool_pages, 2, 64)), ValueError), (dict(page_ids=t["page_ids"][:-1]), ValueError),
                     (dict(page_ids=t["page_ids"].long()), TypeError), (dict(v_new=t["v_new"].transpose(0, 1).contiguous().transpose(0, 1)), ValueError)):
        with pytest.raises(err):
            kvq.forward(p, *args(**bad))
    with pytest.raises(ValueError):
        kvq.forward(p, *args(), launch_events=[])
    with pytest.raises(ValueError):
        kvq.forward(p, *args(), out=torch.empty(1, 4, 64, dtype=torch.bfloat16, device=dev))
    q = kv.plan(kv_len=[20], page_indptr=[0, 2], page_ids=[1, 0], num_kv_heads=2, head_dim=64, num_pool_pages=2, device=dev)
    with pytest.raises(ValueError):
        kvq.kv_export(q, kvq.empty_cache(1, 2, 64, device=dev))
    with pytest.raises(ValueError):
        kvq.kv_export(q, ok, k_packed=torch.empty(19, 2, 64, dtype=torch.bfloat16, device=dev))
    with pytest.raises(ValueError):
        kvq.kv_import(q, torch.empty(20, 2, 64, device=dev), torch.empty(20, 2, 64, device=dev), ok)
