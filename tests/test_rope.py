"""Rotary positions (include/sangam_rope.h, paper_2607_04206_amd/rope.py).

CPU: the rates of every scaling against the formulas, refusals of the C entries
and of the Python calls.
GPU: against the rotation in float64, at every type, layout and kind of stride.

Bar of an element y of a pair (x0, x1), y = m (x0 c - x1 s): the rounding to
its type, at most eps / 2 of |y| (half the smallest subnormal at least), and
m (|x0| + |x1|) times the errors in fp32: sine and cosine to 2 ulp (2^-23
below 1), the reduced angle's rounding (2^-28 turns, 2^-25 rad), the factor m
(2^-24) and the products and sum (2 * 2^-24), together below 2^-21.
"""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2607_04206_amd import _lib, rope

TYPES = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half the smallest subnormal


def rates(rot, base=10000.0, scaling="none", factor=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0, magnitude=None, **_):
    """f_j and m from the formulas, in float64."""
    j = np.arange(rot // 2)
    f = base ** (-2.0 * j / rot)
    m = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "ntk":
        f = (base * factor ** (rot / (rot - 2.0))) ** (-2.0 * j / rot)
    elif scaling == "yarn":
        turns = original_len * f / (2 * math.pi)
        g = np.clip((turns - beta_slow) / (beta_fast - beta_slow), 0, 1)
        f = g * f + (1 - g) * f / factor
        m = 0.1 * math.log(factor) + 1
    return f, m if magnitude is None else magnitude


def rotated(x, positions, rot, interleaved, transpose=False, **scale):
    """x [rows, heads, D] (float64) rotated, and the bar's fp32 part."""
    f, m = rates(rot, **scale)
    angle = np.asarray(positions, np.float64)[:, None, None] * f
    c, s = np.cos(angle) * m, np.sin(angle) * m * (-1 if transpose else 1)
    y, bar = x.copy(), np.zeros_like(x)
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    bar[..., lo] = bar[..., hi] = 2.0 ** -21 * m * (np.abs(x[..., lo]) + np.abs(x[..., hi]))
    return y, bar


# ------------------------------------------------------------------ plan (CPU)
SCALES = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0, base=500000.0),
          dict(scaling="yarn", factor=16.0, original_len=4096.0), dict(scaling="yarn", factor=2.0, original_len=100.0, beta_fast=8.0, beta_slow=0.5),
          dict(magnitude=1.25), dict(scaling="yarn", factor=4.0, original_len=8192.0, magnitude=1.0)]


@pytest.mark.parametrize("rot", [4, 6, 64, 128, 512])
@pytest.mark.parametrize("scale", SCALES)
def test_rates(rot, scale):
    p = rope.plan(rot_dim=rot, **scale)
    f, m = rates(rot, **scale)
    turns = p.host[256:].view(np.float64)
    assert turns.shape == (rot // 2,)
    assert np.allclose(turns, f / (2 * math.pi), rtol=1e-14, atol=0)  # some operations of 2^-53 each, pow() among them
    assert p.host[24:28].view(np.float32)[0] == np.float32(m)


def index_rates(rot, base, original_len, factor, beta_fast=32.0, beta_slow=1.0):
    """f_j of YaRN scaling by index from its formula: the pair's own rate up to index lo, a factor-th from hi on, linear between."""
    at = lambda turns: rot * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    lo = max(0, math.floor(at(beta_fast)))
    hi = rot - 1 if beta_slow == 0 else min(rot - 1, math.ceil(at(beta_slow)))
    j = np.arange(rot // 2)
    share = np.clip((j - lo) / max(hi - lo, 1e-3), 0, 1)  # of the stretched rate
    f = base ** (-2.0 * j / rot)
    return f * (1 - share) + f / factor * share, lo, hi


INDEXED = [dict(rot=128, base=1e6, original_len=32768.0, factor=4.0), dict(rot=128, base=1e4, original_len=4096.0, factor=16.0),
           dict(rot=64, base=5e5, original_len=8192.0, factor=8.0), dict(rot=128, base=1e4, original_len=256.0, factor=2.0),
           dict(rot=32, base=1e4, original_len=4096.0, factor=40.0, beta_fast=8.0, beta_slow=0.0), dict(rot=8, base=1e4, original_len=6.0, factor=3.0)]


@pytest.mark.parametrize("c,lo,hi", zip(INDEXED, (23, 20, 9, 1, 7, 0), (40, 46, 18, 26, 31, 0)))
def test_rates_of_released_checkpoints(c, lo, hi):
    """YaRN scaling as released checkpoints have it: the ramp is linear in the pair's index between two whole numbers."""
    f, *ends = index_rates(**c)
    assert ends == [lo, hi]
    scale = {**c, "rot_dim": c["rot"]}
    del scale["rot"]
    p = rope.plan(scaling="yarn_index", **scale)
    assert np.allclose(p.host[256:].view(np.float64), f / (2 * math.pi), rtol=1e-14, atol=0)
    assert p.host[24:28].view(np.float32)[0] == np.float32(0.1 * math.log(c["factor"]) + 1)
    paper = rope.plan(scaling="yarn", **scale).host[256:].view(np.float64) * 2 * math.pi
    same = np.isclose(paper, f, rtol=1e-12, atol=0)
    if c["rot"] > 32:  # (pairs up to lo keep their rates in both; over 6 positions none of the paper's does)
        assert same[:lo + 1].all() and not same.all()
    if c == INDEXED[0]:
        assert (~same).sum() == 16 and (paper / f).min() == pytest.approx(0.58, abs=0.01)


@pytest.mark.parametrize("original_len", [1e9, 1e12])
def test_yarn_by_index_of_long_lengths(original_len):
    """Where every pair turns more than beta_fast times, all keep their rates."""
    p = rope.plan(rot_dim=64, scaling="yarn_index", factor=4.0, original_len=original_len)
    assert np.allclose(p.host[256:].view(np.float64), rates(64)[0] / (2 * math.pi), rtol=1e-14, atol=0)


def test_yarn_by_index_refuses():
    for bad in (dict(original_len=0.0), dict(original_len=1e-3), dict(beta_slow=32.0), dict(beta_slow=-1.0), dict(factor=0.5), dict(original_len=float("nan"))):
        with pytest.raises(_lib.SangamError) as e:
            rope.plan(rot_dim=64, scaling="yarn_index", **{**dict(factor=2.0, original_len=4096.0), **bad})
        assert e.value.status == -1 and str(e.value)


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=514), dict(rot_dim=-2), dict(base=1.0), dict(base=float("nan")),
                                 dict(base=float("inf")), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")),
                                 dict(scaling="ntk", factor=2.0, rot_dim=2), dict(scaling="yarn", factor=2.0),
                                 dict(scaling="yarn", factor=2.0, original_len=64.0, beta_fast=1.0, beta_slow=1.0),
                                 dict(scaling="yarn", factor=2.0, original_len=64.0, beta_slow=-1.0), dict(magnitude=float("inf"))])
def test_plan_refuses(bad):
    with pytest.raises(_lib.SangamError) as e:
        rope.plan(**{**dict(rot_dim=64), **bad})
    assert e.value.status == -1 and str(e.value)


def test_plan_refuses_in_python_and_by_size():
    for bad in (dict(scaling="cubic"), dict(magnitude=0.0), dict(magnitude=-1.0)):
        with pytest.raises(ValueError):
            rope.plan(rot_dim=64, **bad)
    d = _lib.RopeDesc(64, 0, 0, 0, 10000.0)
    used = ctypes.c_size_t(0)
    f = _lib.lib.sangam_rope_plan
    assert f(ctypes.byref(d), None, 0, ctypes.byref(used)) == -5 and used.value == 256 + 32 * 8
    assert f(None, None, 0, ctypes.byref(used)) == -1 and f(ctypes.byref(d), None, 0, None) == -1
    d.scaling = 9
    assert f(ctypes.byref(d), None, 0, ctypes.byref(used)) == -1
    d.scaling, d.interleaved = 0, 2
    assert f(ctypes.byref(d), None, 0, ctypes.byref(used)) == -1


def test_entries_without_memory(tmp_path, monkeypatch):
    """An exception in a C entry becomes a status of its own and a message, and plan() takes it for no size."""
    if shutil.which("g++"):
        exe = str(tmp_path / "driver")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(os.path.dirname(os.path.abspath(__file__)), "sanitize", "entry_driver.cpp"),
                        "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout
    monkeypatch.setattr(rope.lib, "sangam_rope_plan", lambda *a: -9)
    with pytest.raises(_lib.SangamError) as e:
        rope.plan(rot_dim=64)
    assert e.value.status == -9


def _tensor(**over):
    t = dict(in_=4096, out=4096, in_row_stride=256, in_head_stride=64, out_row_stride=256, out_head_stride=64, heads=4, reserved=0)
    t.update(over)
    return _lib.RopeTensor(*[t[n] for n, _ in _lib.RopeTensor._fields_])


@pytest.mark.parametrize("over,call,status", [
    (dict(), dict(plan=None), -8), (dict(), dict(q=None), -1), (dict(), dict(dtype=3), -2), (dict(), dict(head_dim=32), -1),
    (dict(), dict(head_dim=1024), -1), (dict(), dict(rows=-1), -1), (dict(), dict(rows=1 << 31), -1), (dict(), dict(transpose=2), -1),
    (dict(), dict(positions=None), -1), (dict(), dict(plan_dev=None), -1), (dict(), dict(plan_dev=4104), -6), (dict(), dict(positions=4098), -6),
    (dict(in_=None), {}, -1), (dict(out=None), {}, -1), (dict(in_=4097, out=1 << 20), {}, -6), (dict(heads=0), {}, -1),
    (dict(in_row_stride=-256, out=1 << 20), {}, -1), (dict(out_row_stride=-256, in_row_stride=-256), {}, -1),
    (dict(out=1 << 20, out_head_stride=63), {}, -1), (dict(out=1 << 20, out_row_stride=255), {}, -1), (dict(out=1 << 20, out_row_stride=0), {}, -1),
    (dict(in_row_stride=1 << 40, out_row_stride=1 << 40), dict(rows=(1 << 31) - 1), -1),  # more than 64 bits hold
    (dict(out_row_stride=512), {}, -1)])  # in place with other strides
def test_rotate_refuses(over, call, status):
    # fake device addresses: every check fails before any HIP call
    p = rope.plan(rot_dim=64)
    a = dict(plan=p.host_ptr(), plan_dev=4096, q=ctypes.byref(_tensor(**over)), head_dim=64, dtype=0, positions=4096, rows=10, transpose=0)
    a.update(call)
    got = _lib.lib.sangam_rope_rotate(a["plan"], a["plan_dev"], a["q"], None, a["head_dim"], a["dtype"], a["positions"], a["rows"], a["transpose"], None)
    assert got == status and _lib.lib.sangam_last_error()


def test_no_rows_is_no_launch():
    p = rope.plan(rot_dim=64)
    q = _tensor(in_=None, out=None)
    assert _lib.lib.sangam_rope_rotate(p.host_ptr(), None, ctypes.byref(q), ctypes.byref(q), 64, 0, None, 0, 0, None) == 0


@pytest.mark.parametrize("seed", [1, 2])
def test_plan_under_asan_ubsan(tmp_path, seed):
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "driver")
    csrc = os.path.join(os.path.dirname(here), "paper_2607_04206_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1", "-Wall",
                    os.path.join(here, "sanitize", "rope_driver.cpp"), os.path.join(csrc, "rope_plan.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe, str(seed)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and " 0 failed checks" in r.stdout, r.stdout[-500:] + r.stderr[-2000:]
    assert int(r.stdout.split()[0]) > 2000 and int(r.stdout.split()[2]) > 2000


def _refused(q_in, q_out, k_in=None, k_out=None):
    """Whether the C entry refuses tensors for their overlaps (of host tensors:
    what passes the checks fails for the missing plan_dev, in another way)."""
    p = rope.plan(rot_dim=8)
    c = [_lib.RopeTensor(i.data_ptr(), o.data_ptr(), i.stride(0), i.stride(1), o.stride(0), o.stride(1), i.shape[1], 0)
         for i, o in ((q_in, q_out), (k_in, k_out)) if i is not None]
    st = _lib.lib.sangam_rope_rotate(p.host_ptr(), None, ctypes.byref(c[0]), ctypes.byref(c[1]) if len(c) > 1 else None, 8, 2, 4096,
                                     q_in.shape[0], 0, None)
    assert st == -1
    return b"overlap" in _lib.lib.sangam_last_error()


def test_overlaps_are_refused():
    x, y = torch.zeros(10, 6, 8), torch.zeros(10, 6, 8)
    assert not _refused(x, x) and not _refused(x, y) and not _refused(x[:, :2], x[:, 2:4]) and not _refused(x[:, 2:4], x[:, :2])
    assert not _refused(x[:5], x[5:]) and not _refused(x[:, :3], x[:, :3], x[:, 3:], x[:, 3:])
    assert _refused(x[:, :2], x[:, 1:3]) and _refused(x[:5], x[4:9]) and _refused(x[:9], x[1:]) and _refused(x[1:], x[:9])
    assert _refused(x[:9, 4:6], x[1:, 4:6]) and not _refused(x[:9, 4:6], x[1:, :2])
    assert _refused(x[:, :2], y[:, :2], x[:, 2:3], y[:, 1:2]) and _refused(x[:, :2], y[:, :2], x[:, 2:3], x[:, :1])
    assert _refused(x.transpose(0, 1).contiguous().transpose(0, 1), x[:, :6], x, x) and not _refused(x[:1], y[:1], x[1:2], y[1:2])


def test_strides_of_single_rows_and_heads_are_not_read():
    # what passes the checks of the tensors fails for the missing plan_dev
    p = rope.plan(rot_dim=64)

    def call(rows, **over):
        st = _lib.lib.sangam_rope_rotate(p.host_ptr(), None, ctypes.byref(_tensor(**over)), None, 64, 0, 4096, rows, 0, None)
        return st, b"plan_dev" in _lib.lib.sangam_last_error()
    for stride in (0, 3, 999, -1, 1 << 60):
        assert call(1, out_row_stride=stride) == call(1, in_row_stride=stride) == (-1, True)
        assert call(10, heads=1, out_head_stride=stride) == call(10, heads=1, in_head_stride=stride) == (-1, True)
        assert call(10, out_row_stride=stride)[1] == call(10, in_head_stride=stride)[1] is False
    x = torch.zeros(10, 6, 8)
    assert not _refused(x[:1], x[:1].reshape(1, 48).view(1, 6, 8)) and _refused(x[:1, :4], x[:1, 2:6]) and not _refused(x[:1, :3], x[:1, 3:])


# ------------------------------------------------------------------------ GPU
@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    return torch.device("cuda:0")


def check(got, x, positions, rot, interleaved, **kw):
    want, bar = rotated(x.double().cpu().numpy(), positions.cpu().numpy(), rot, interleaved, **kw)
    bar += np.maximum(torch.finfo(x.dtype).eps / 2 * (np.abs(want) + bar), TYPES[x.dtype])
    bar[..., rot:] = 0.0  # passes unchanged
    d = np.abs(got.double().cpu().numpy() - want)
    bad = np.flatnonzero((d > bar).reshape(-1))
    if len(bad):
        at = np.unravel_index(bad[0], d.shape)
        pytest.fail(f"{len(bad)} of {d.size} off, the first at {at}: {got[at].item()}, not {want[at]} to {bar[at]:.2e}", pytrace=False)


def inputs(rows, hq, hkv, d, dtype, dev, seed=0, far=10000):
    g = torch.Generator(device=dev).manual_seed(seed + rows)
    draw = lambda h: torch.randn(rows, h, d, generator=g, device=dev).to(dtype)  # noqa: E731
    return draw(hq), draw(hkv), torch.randint(0, far, (rows,), generator=g, device=dev, dtype=torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hkv,d,rot", [(1, 32, 32, 128, 128), (5, 1, 1, 64, 64), (33, 28, 4, 128, 64), (130, 8, 2, 64, 16), (7, 3, 1, 256, 192),
                                               (6, 5, 2, 100, 34), (3, 2, 2, 64, 2), (2, 4, 1, 512, 512), (3000, 4, 4, 64, 48), (9, 3, 2, 80, 80), (11, 3, 2, 37, 24)])
def test_shapes(dev, dtype, interleaved, rows, hq, hkv, d, rot):
    print(f"[case] rope {dtype} {interleaved} {rows} rows {hq}/{hkv} of {d}, {rot} rotate", flush=True)
    q, k, pos = inputs(rows, hq, hkv, d, dtype, dev)
    keep = q.clone(), k.clone()
    p = rope.plan(rot_dim=rot, interleaved=interleaved, device=dev)
    for transpose in (False, True):
        for got, x in zip(rope.rotate(p, q, k, pos, transpose=transpose), keep):
            check(got, x, pos, rot, interleaved, transpose=transpose)
    assert torch.equal(q, keep[0]) and torch.equal(k, keep[1])


@pytest.mark.gpu
@pytest.mark.parametrize("scale", SCALES)
def test_scalings_at_far_positions(dev, scale):
    q, k, _ = inputs(12, 4, 2, 128, torch.float32, dev)
    pos = torch.tensor([0, 1, 2, 31, -1, -77, 4095, 131071, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=dev)
    p = rope.plan(rot_dim=128, device=dev, **scale)
    # the oracle's own angle, p f in float64, is off by 2^-53 of itself, more than the bar from 2^28 rad on: compared below it
    near = pos.cpu().numpy() < 2 ** 28
    near &= pos.cpu().numpy() > -2 ** 28
    for got, x in zip(rope.rotate(p, q, k, pos), (q, k)):
        check(got[torch.from_numpy(near).to(dev)], x[torch.from_numpy(near).to(dev)], pos[torch.from_numpy(near).to(dev)], 128, False, **scale)
        assert torch.isfinite(got).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", SCALES)
def test_furthest_positions(dev, scale):
    """Positions from 2^28 on, whose angles in float64 are off by more than the bar of an element allows, against 80-bit ones.
    Errors of an angle, in 2^-53 of itself: pow() 2, the constant 2 pi 0.4, the quotient by it 1, the product with the position 1,
    and a factor 1: below 8. NTK's base adds 5.1 (its power of the factor 4.1, its product 1): below 16. YaRN's share g is off
    by up to 3.3 times turns / (beta_fast - beta_slow), at most 1.1, and f by the factor times that where g is small: below 8 factors."""
    if np.finfo(np.longdouble).nmant < 63:
        pytest.skip("needs an 80-bit long double")
    q, k, _ = inputs(7, 4, 2, 128, torch.float32, dev)
    pos = torch.tensor([1 << 28, (1 << 28) + 1, (1 << 30) - 7, 2 ** 31 - 1, -2 ** 31, -2 ** 29 - 3, 1234567891], dtype=torch.int32, device=dev)
    p = rope.plan(rot_dim=128, device=dev, **scale)
    L, kind, s = np.longdouble, scale.get("scaling", "none"), scale.get("factor", 1.0)
    two_pi, j = 8 * np.arctan(L(1)), np.arange(64, dtype=L)
    base = L(scale.get("base", 10000.0)) * (L(s) ** (L(128) / 126) if kind == "ntk" else 1)
    f, m = base ** (-2 * j / 128), L(scale.get("magnitude") or (1 + L(0.1) * np.log(L(s)) if kind == "yarn" else 1))
    if kind == "linear":
        f = f / L(s)
    elif kind == "yarn":
        fast, slow = L(scale.get("beta_fast", 32.0)), L(scale.get("beta_slow", 1.0))
        g = np.clip((L(scale["original_len"]) * f / two_pi - slow) / (fast - slow), 0, 1)
        f = g * f + (1 - g) * f / L(s)
    angle = pos.cpu().numpy().astype(L)[:, None, None] * f
    off = 2.0 ** -53 * {"ntk": 16, "yarn": 8 * s}.get(kind, 8) * np.abs(angle).astype(np.float64)
    for got, x in zip(rope.rotate(p, q, k, pos), (q, k)):
        x = x.double().cpu().numpy()
        lo, hi = x[..., :64], x[..., 64:]
        c, t = np.cos(angle) * m, np.sin(angle) * m
        want = np.concatenate([lo * c - hi * t, hi * c + lo * t], -1).astype(np.float64)
        bar = np.tile(float(m) * (np.abs(lo) + np.abs(hi)) * (2.0 ** -21 + off), 2) + 2.0 ** -24 * np.abs(want)
        assert (np.abs(got.double().cpu().numpy() - want) <= bar).all()
        assert off[:, :, 32:].max() < 2.0 ** -22 * (4 * s if kind == "yarn" else 1)  # half of the pairs to 2^-22 rad


@pytest.mark.gpu
def test_yarn_by_index(dev):
    """To the bar of an element (above), in fp32."""
    c = INDEXED[1]
    q, k, pos = inputs(40, 4, 2, 128, torch.float32, dev, far=65536)
    p = rope.plan(rot_dim=128, scaling="yarn_index", base=c["base"], original_len=c["original_len"], factor=c["factor"], device=dev)
    m = 0.1 * math.log(c["factor"]) + 1
    angle = pos.cpu().numpy()[:, None, None] * index_rates(**c)[0]
    for got, x in zip(rope.rotate(p, q, k, pos), (q, k)):
        x = x.double().cpu().numpy()
        z = (x[..., :64] + 1j * x[..., 64:]) * np.exp(1j * angle) * m
        want = np.concatenate([z.real, z.imag], -1)
        bar = 2.0 ** -21 * m * np.tile(np.abs(x[..., :64]) + np.abs(x[..., 64:]), 2) + 2.0 ** -24 * np.abs(want)
        assert (np.abs(got.double().cpu().numpy() - want) <= bar).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (64, 30)])
def test_views_in_place(dev, dtype, interleaved, d, rot):
    """q and k inside a fused projection's output, rotated in place: its other
    columns and the rows behind keep their bits."""
    rows, hq, hkv = 70, 6, 2
    g = torch.Generator(device=dev).manual_seed(3)
    x = torch.randn(rows + 9, hq + 2 * hkv, d, generator=g, device=dev).to(dtype)
    pos = torch.randint(0, 5000, (rows,), generator=g, device=dev, dtype=torch.int32)
    keep = x.clone()
    p = rope.plan(rot_dim=rot, interleaved=interleaved, device=dev)
    q, k = x[:rows, :hq], x[:rows, hq:hq + hkv]
    got = rope.rotate(p, q, k, pos, q_out=q, k_out=x[:rows, hq:hq + hkv])
    assert got[0] is q
    check(q, keep[:rows, :hq], pos, rot, interleaved)
    check(k, keep[:rows, hq:hq + hkv], pos, rot, interleaved)
    assert torch.equal(x[:, hq + hkv:], keep[:, hq + hkv:]) and torch.equal(x[rows:], keep[rows:])


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides(dev, interleaved):
    """Head-major inputs and outputs, broadcast inputs, addresses off 16 bytes."""
    rows, h, d = 37, 5, 64
    q, k, pos = inputs(rows, h, 2, d, torch.bfloat16, dev)
    p = rope.plan(rot_dim=d, interleaved=interleaved, device=dev)
    want = rope.rotate(p, q, k, pos)
    major = q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty_like(major.transpose(0, 1).contiguous()).transpose(0, 1)
    assert torch.equal(rope.rotate(p, major, None, pos, q_out=out)[0], want[0])
    buf = torch.zeros(rows * h * d + 1, dtype=torch.bfloat16, device=dev)
    odd = buf[1:].view(rows, h, d)
    odd.copy_(q)
    for got, w in zip(rope.rotate(p, odd, k, pos, q_out=odd), want):
        assert torch.equal(got, w)
    assert buf[0] == 0
    one = q[:, :1].expand(rows, 4, d)
    got, none = rope.rotate(p, one, None, pos)
    assert none is None and torch.equal(got, want[0][:, :1].expand(rows, 4, d))
    same_row = q[:1].expand(rows, h, d)
    check(rope.rotate(p, same_row, None, pos)[0], same_row, pos, d, interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_single_rows_and_heads(dev, interleaved):
    """Their odd strides change nothing, in place either."""
    for rows, h in ((1, 6), (40, 1), (1, 1)):
        q, k, pos = inputs(rows, h, h, 128, torch.bfloat16, dev)
        p = rope.plan(rot_dim=128, interleaved=interleaved, device=dev)
        want = rope.rotate(p, q, k, pos)
        strides = (13 if rows == 1 else h * 128, 7 if h == 1 else 128, 1)
        odd = [x.as_strided(x.shape, strides) for x in (q, k)]
        assert all(torch.equal(a, b) for a, b in zip(rope.rotate(p, *odd, pos), want))
        rope.rotate(p, q, k, pos, q_out=odd[0], k_out=odd[1])
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 126), (128, 110), (128, 122), (64, 46), (37, 24), (20, 18), (64, 62), (21, 16), (130, 128), (24, 8), (9, 8), (7, 4)])
def test_numbers_of_pairs_that_no_vector_divides(dev, dtype, interleaved, d, rot):
    """Outputs beside guards, head strides and addresses of odd numbers of
    elements, and the same in place, which gives the same bits."""
    rows, h, pad = 53, 5, 3
    q, k, pos = inputs(rows, h, 2, d, dtype, dev)
    p = rope.plan(rot_dim=rot, interleaved=interleaved, device=dev)
    buf = torch.full((1 + rows * h * (d + pad),), 7.0, dtype=dtype, device=dev)
    out = buf[1:].view(rows, h, d + pad)[:, :, :d]
    got = rope.rotate(p, q, k, pos, q_out=out)
    check(out, q, pos, rot, interleaved)
    check(got[1], k, pos, rot, interleaved)
    guards = buf.clone()
    guards[1:].view(rows, h, d + pad)[:, :, :d] = 7.0
    assert (guards == 7.0).all()
    here = buf.clone()
    x = here[1:].view(rows, h, d + pad)[:, :, :d]
    x.copy_(q)
    apart = rope.rotate(p, x, k, pos, q_out=x)[1]  # q in place, k not
    assert torch.equal(here, buf) and torch.equal(apart, got[1])
    both = k.clone()
    x.copy_(q)
    rope.rotate(p, x, both, pos, q_out=x, k_out=both)
    assert torch.equal(here, buf) and torch.equal(both, got[1])


@pytest.mark.gpu
def test_rows_far_apart(dev):
    """Offsets past 2^31 elements and 2^32 bytes."""
    d, step = 64, 2 ** 31 + 64
    buf = torch.empty(step + 4 * d, dtype=torch.bfloat16, device=dev)
    q, k, pos = inputs(2, 2, 1, d, torch.bfloat16, dev)
    far = buf.as_strided((2, 2, d), (step, d, 1))
    far.copy_(q)
    p = rope.plan(rot_dim=d, device=dev)
    want = rope.rotate(p, q, k, pos)
    got = rope.rotate(p, far, k, pos, q_out=far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_gradient(dev):
    """The transpose against the formula (<g, R x> = <R' g, x>) and against
    differences of the rotation, a YaRN magnitude included. In fp32 an element
    errs by 2^-21 m (|x0| + |x1|) + 2^-24 |y|."""
    scale = dict(scaling="yarn", factor=8.0, original_len=256.0)
    q, k, pos = inputs(9, 3, 2, 64, torch.float32, dev, far=4096)
    gq, gk, _ = inputs(9, 3, 2, 64, torch.float32, dev, seed=50)
    for interleaved in (False, True):
        p = rope.plan(rot_dim=48, interleaved=interleaved, device=dev, **scale)
        y, dx = rope.rotate(p, q, k, pos), rope.rotate(p, gq, gk, pos, transpose=True)
        for x, g, a, b in zip((q, k), (gq, gk), y, dx):
            check(b, g, pos, 48, interleaved, transpose=True, **scale)
            left, right = (g.double() * a.double()).sum(), (b.double() * x.double()).sum()
            m = 0.1 * math.log(8.0) + 1
            assert abs(left - right) <= 4 * 2.0 ** -21 * m * (g.double().abs().sum() * x.double().abs().max())
            for at in ((0, 0, 0), (3, 1, 20), (8, 0, 47), (5, 1, 60)):
                step = torch.zeros_like(x)
                step[at] = 0.5
                ends = [rope.rotate(p, x + s * step, None, pos)[0].double() for s in (1, -1)]
                slope = ((ends[0] - ends[1]) * g.double()).sum()  # the ends are 1 apart, and the rotation is linear
                row = at[0]
                bar = 2 * 2.0 ** -21 * m * 2 * (x[row].abs().max() + 0.5).double() * g[row].double().abs().sum() * 2
                assert abs(slope - b[at].double()) <= bar


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("transpose", [False, True])
def test_autograd(dev, dtype, transpose):
    """Outputs are the bits of a call without gradients, and q and k get the transpose's: to its bar (above) from the formula, for
    gradients in any layout, of one tensor or both."""
    q, k, pos = inputs(33, 4, 2, 64, dtype, dev)
    gq, gk, _ = inputs(33, 4, 2, 64, dtype, dev, seed=50)
    p = rope.plan(rot_dim=48, device=dev)
    want = rope.rotate(p, q, k, pos, transpose=transpose)
    assert not want[0].requires_grad
    q.requires_grad_(), k.requires_grad_()
    with torch.no_grad():
        assert not rope.rotate(p, q, k, pos, transpose=transpose)[0].requires_grad
    for stream in (None, torch.cuda.Stream(dev)):
        torch.cuda.synchronize()
        out = rope.rotate(p, q, k, pos, transpose=transpose, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        wide = torch.stack([gq, gq], -1)[..., 0]  # dims two elements apart
        for grads in ((gq, gk), (wide, gk)):
            for d, g in zip(torch.autograd.grad(out, (q, k), grads, retain_graph=True), (gq, gk)):
                check(d, g, pos, 48, False, transpose=not transpose)
        d, none = torch.autograd.grad(out[0], (q, k), gq, retain_graph=True, allow_unused=True)
        check(d, gq, pos, 48, False, transpose=not transpose)
        assert none is None
        check(torch.autograd.grad(out[1], k, gk)[0], gk, pos, 48, False, transpose=not transpose)
    # one tensor that requires none, one alone, none of the rows
    out = rope.rotate(p, q.detach(), k, pos, transpose=transpose)
    assert not out[0].requires_grad
    check(torch.autograd.grad(out[1], k, gk)[0], gk, pos, 48, False, transpose=not transpose)
    out = rope.rotate(p, q, None, pos, transpose=transpose)
    assert out[1] is None
    ones = torch.ones_like(gq)
    check(torch.autograd.grad(out[0].sum(), q)[0], ones, pos, 48, False, transpose=not transpose)  # (an expanded gradient)
    assert torch.autograd.grad(rope.rotate(p, q[:0], None, pos[:0])[0].sum(), q)[0].abs().max() == 0
    # views of one projection, and the gradient's own gradient
    x = torch.cat([q, k, k], 1).detach().requires_grad_()
    a, b = rope.rotate(p, x[:, :4], x[:, 4:6], pos, transpose=transpose)
    dx, = torch.autograd.grad((a * gq).sum() + (b * gk).sum(), x)
    check(dx[:, :4], gq, pos, 48, False, transpose=not transpose)
    check(dx[:, 4:6], gk, pos, 48, False, transpose=not transpose)
    assert not dx[:, 6:].any()
    g = gq.clone().requires_grad_()
    dq, = torch.autograd.grad(rope.rotate(p, q, None, pos, transpose=transpose)[0], q, g, create_graph=True)
    check(torch.autograd.grad(dq, g, gq)[0], gq, pos, 48, False, transpose=transpose)
    for kw in (dict(q_out=torch.empty_like(q)), dict(k_out=k.detach()), dict(q_out=q, k_out=k)):
        with pytest.raises(ValueError, match="gradients"):
            rope.rotate(p, q, k, pos, **kw)
    with torch.no_grad():
        rope.rotate(p, q, k, pos, q_out=torch.empty_like(q))


@pytest.mark.gpu
def test_refusals_with_gradients(dev):
    """The words of a call without them."""
    q, k, pos = inputs(10, 4, 2, 64, torch.bfloat16, dev)
    p = rope.plan(rot_dim=64, device=dev)
    q.requires_grad_()
    for err, a, words in ((TypeError, (q, k, pos.tolist()), "positions"), (TypeError, (q, k, None), "positions"), (ValueError, (q, k, pos[:9]), "positions"),
                          (TypeError, (q, k.float(), pos), "k must"), (TypeError, (q, [k], pos), "k must"), (ValueError, (q, k[..., :32], pos), "k must")):
        with pytest.raises(err, match=words):
            rope.rotate(p, *a)


@pytest.mark.gpu
def test_autograd_in_a_graph(dev):
    """Forward and backward captured together, replayed at other positions."""
    q, k, pos = inputs(50, 4, 2, 64, torch.bfloat16, dev)
    gq, gk, _ = inputs(50, 4, 2, 64, torch.bfloat16, dev, seed=50)
    p = rope.plan(rot_dim=64, device=dev)
    s = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):  # leaves that only this stream knows
        leaves = [x.clone().requires_grad_() for x in (q, k)]
        torch.autograd.grad(rope.rotate(p, *leaves, pos), leaves, (gq, gk))
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = rope.rotate(p, *leaves, pos)
        grads = torch.autograd.grad(out, leaves, (gq, gk))
    for _ in range(4):
        pos.add_(17)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = rope.rotate(p, q, k, pos), rope.rotate(p, gq, gk, pos, transpose=True)
        assert all(torch.equal(a, b) for a, b in zip((*out, *grads), (*want[0], *want[1])))


@pytest.mark.gpu
def test_streams_and_graphs(dev):
    q, k, pos = inputs(100, 8, 2, 128, torch.bfloat16, dev)
    p = rope.plan(rot_dim=128, device=dev)
    want = rope.rotate(p, q, k, pos)
    s = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    got = rope.rotate(p, q, k, pos, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = [torch.empty_like(x) for x in (q, k)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        rope.rotate(p, q, k, pos, q_out=out[0], k_out=out[1])
    for n in range(4):
        pos.add_(17)
        for o in out:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = rope.rotate(p, q, k, pos)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.gpu
def test_memory_between_streams(dev):
    """Outputs of a call on a given stream do not take memory that the current
    stream still reads, and a plan's memory outlives the call that reads it."""
    q, _, pos = inputs(300, 16, 2, 64, torch.bfloat16, dev)
    p = rope.plan(rot_dim=64, device=dev)
    want, _ = rope.rotate(p, q, None, pos)
    s = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    held = torch.full_like(want, 3.0)
    torch.cuda._sleep(20_000_000)  # the copy of `held` is still to come when its memory is free
    copy = held.clone()
    del held
    got, _ = rope.rotate(p, q, None, pos, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(copy, torch.full_like(want, 3.0))
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        got, _ = rope.rotate(p, q, None, pos)
    size = p.dev.numel()
    del p
    others = [torch.zeros(size, dtype=torch.uint8, device=dev) for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 8


@pytest.mark.gpu
def test_python_refusals(dev):
    q, k, pos = inputs(10, 4, 2, 64, torch.bfloat16, dev)
    p = rope.plan(rot_dim=64, device=dev)
    fused = torch.zeros(10, 8, 64, dtype=torch.bfloat16, device=dev)
    for err, a, kw in ((TypeError, (q.double(), k, pos), {}), (TypeError, (q, k.float(), pos), {}), (TypeError, (q, k, pos.long()), {}),
                       (ValueError, (q, k, pos[:9]), {}), (ValueError, (q[:9], k, pos), {}), (ValueError, (q, k, pos.cpu()), {}),
                       (ValueError, (q, k[..., :32], pos), {}), (ValueError, (q.transpose(1, 2).contiguous().transpose(1, 2), k, pos), {}),
                       (ValueError, (q, k, pos), dict(q_out=k)), (ValueError, (q, k, pos), dict(q_out=q[:9])), (ValueError, (q, None, pos), dict(k_out=k)),
                       (_lib.SangamError, (fused[:, :4], fused[:, 4:6], pos), dict(q_out=fused[:, 2:6])), (TypeError, (q, k[0], pos), {}),
                       (_lib.SangamError, (q, k, pos), dict(q_out=fused[:, :4], k_out=fused[:, 3:5])), (TypeError, (None, k, pos), {}),
                       (ValueError, (q.cpu(), k.cpu(), pos.cpu()), {})):
        with pytest.raises(err):
            rope.rotate(p, *a, **kw)
    with pytest.raises(_lib.SangamError):
        rope.rotate(rope.plan(rot_dim=128, device=dev), q, k, pos)
    with pytest.raises(_lib.SangamError):
        rope.rotate(p, q, k, pos, q_out=torch.empty(1, 1, 64, dtype=q.dtype, device=dev).expand(10, 4, 64))
    empty = rope.rotate(p, q[:0], k[:0], pos[:0])
    assert empty[0].shape == (0, 4, 64)
