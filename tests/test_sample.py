"""Sampling (include/sangam_sample.h, paper_2607_04206_amd/sample.py) against its
definition in 64 bits on the host: filters and draws by rank order, confidences,
ties, masked and infinite logits, odd sizes and strides, parameters a row or a
request, refusals."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2607_04206_amd import _lib, sample

INF = math.inf
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def ranked(x, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """Tokens in rank order, the weights of the kept ones (0 behind them) and (x - X) / T of each; None: a row with nothing."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -INF, x)
    if x.max() == INF:
        x = np.where(x == INF, 0.0, -INF)
    if x.max() == -INF:
        return None
    order = np.argsort(-x, kind="stable")
    with np.errstate(invalid="ignore", over="ignore"):
        z = (x[order] - x.max()) / (temperature if temperature > 0 else 1.0)
    z = np.where(x[order] == -INF, -INF, z)
    w = np.exp(z)
    n = np.arange(len(x))
    if top_k > 0:
        w = np.where(n < top_k, w, 0.0)
    keep = np.cumsum(w) - w < top_p * w.sum() if top_p < 1 else np.ones(len(x), bool)
    if min_p > 0:
        keep &= z >= math.log(min_p)
    return order, np.where(keep | (n == 0), w, 0.0), z


def check(x, token, conf, u, temperature, kind, top_k=0, top_p=1.0, min_p=0.0, forbid=-1):
    """One row's answer against the definition. Tokens are equal, but where the draw falls within 1e-9 of the border to the
    token that came (weights are held to 2^-33, sums to 2^-44 of the largest weight a bin). Confidences: one rounding to 32 bits
    (2^-24 of the value), weights to 2^-33, which the margin's difference and the entropy's factors (|t| up to 64 ln 2) keep as
    2^-32 and 2^-27; where nothing filters and T is 0, weights in 32 bits: 2^-23 (1 + ln(2) |t|) each, weighted sums of |t| are
    under log2(vocab) + 2 times the weights: 2^-19 at 2^18 tokens, and for the entropy that times 2 + log(vocab)."""
    x = np.array(x, np.float64)
    if forbid >= 0:
        x[forbid] = -INF
    got = ranked(x, temperature, top_k, top_p, min_p)
    if got is None:
        assert (token, conf) == (-1, 0.0)
        return
    order, w, z = got
    total = w.sum()
    place = int(np.flatnonzero(order == token)[0])
    if temperature == 0:
        assert place == 0, (token, order[0])
    else:
        up_to = np.cumsum(w)
        target = min(max(u, 0.0), 1.0) * total
        last = int((w > 0).sum()) - 1
        want = min(int(np.searchsorted(up_to, target, side="right")), last)
        if place != want:
            border = up_to[min(place, want)]
            assert w[place] > 0 and abs(border - target) <= 1e-9 * total and abs(place - want) <= max(1, int((w[min(place, want):max(place, want)] <= 1e-9 * total).sum()) + 1), \
                (token, order[want], place, want, border / total, target / total)
    if kind == "probability":
        ref = w[place] / total
    elif kind == "margin":
        ref = (w[0] - (w[1] if len(w) > 1 else 0.0)) / total
    else:
        kept = w > 0
        ref = float((w[kept] * z[kept]).sum() / total - math.log(total))
    plain = temperature == 0 and not (0 < top_k < len(x)) and top_p >= 1 and min_p <= 0
    if plain:
        bar = 2.0 ** -19 * ((2 + math.log(len(x))) if kind == "entropy" else w[0] / total)
    else:
        bar = 2.0 ** -24 * (1 + 2.0 ** -6) * abs(ref) + {"probability": 2.0 ** -33 * w[place] / total, "margin": 2.0 ** -32, "entropy": 2.0 ** -27}[kind]
    assert abs(conf - ref) <= bar, (kind, conf, ref, abs(conf - ref) / bar)


def make(shape, how, dtype, gen):
    rows, vocab = shape
    n = lambda: torch.randn(shape, generator=gen)  # noqa: E731
    if how == "normal":
        x = 2.5 * n()
    elif how == "peaked":
        x = 2.0 * n()
        x.scatter_(1, torch.randint(0, vocab, (rows, 8), generator=gen), 14.0 + n()[:, :1].expand(rows, 8))
    elif how == "equal":
        x = torch.full(shape, -3.25)
    elif how == "near":  # within a bin or two of weights
        x = 5.0 + 1e-3 * n()
    elif how == "ties":
        x = torch.round(2 * n())
    elif how == "zeros":  # of both signs, among others
        x = torch.where(n() > 0, 0.0, -0.0) - (n() > 1).float()
    elif how == "wide":
        x = n() * 10 ** (8 * torch.rand(shape, generator=gen) - 4 if dtype is torch.float16 else 60 * torch.rand(shape, generator=gen) - 25)
    elif how == "masked":
        x = torch.where(torch.rand(shape, generator=gen) < 0.9, -INF, 3 * n())
    elif how == "holes":
        x = 3 * n()
        x = torch.where(torch.rand(shape, generator=gen) < 0.2, math.nan, x)
        x = torch.where(torch.rand(shape, generator=gen) < 0.2, -INF, x)
        x[0] = -INF
        if rows > 1:
            x[1] = math.nan
        if rows > 2:
            x[2] = torch.where(torch.rand((vocab,), generator=gen) < 0.3, INF, x[2])
        if rows > 3:
            x[3] = torch.finfo(dtype).min
    elif how == "rising":
        x = torch.linspace(-20, 12, vocab).expand(shape) + 0.01 * n()
    return x.to(dtype)


PARAMS = [dict(temperature=0.0), dict(temperature=1.0), dict(temperature=0.7, top_k=40), dict(temperature=1.3, top_p=0.9), dict(temperature=0.9, min_p=0.05),
          dict(temperature=0.8, top_k=200, top_p=0.95, min_p=0.02), dict(temperature=0.0, top_p=0.5), dict(temperature=3.0, top_k=3, top_p=0.99),
          dict(temperature=0.05), dict(temperature=INF, top_p=0.25), dict(temperature=1e-30), dict(temperature=1.0, top_p=0.0), dict(temperature=2.0, min_p=1.0),
          dict(temperature=1.0, top_k=1), dict(temperature=1.0, top_k=10 ** 6, top_p=0.5)]


def run_rows(logits, u, params, kind, dev, forbid=-1, **more):
    """Rows of a host tensor on the device, each against the definition."""
    t = logits.to(dev) if not logits.is_cuda else logits
    there = {k: v.to(dev) if torch.is_tensor(v) else v for k, v in params.items()}
    tokens, conf = sample.tokens(t, u.to(dev), confidence=kind, forbid=forbid, **there, **more)
    torch.cuda.synchronize()
    for r, x in enumerate(logits.double().cpu().numpy()):
        one = {k: (float(v[r]) if torch.is_tensor(v) else (float(np.float32(v)) if k != "top_k" else v)) for k, v in params.items()}
        check(x, int(tokens[r]), float(conf[r]), float(u[r]), kind=kind, forbid=forbid, **{k: (int(v) if k == "top_k" else v) for k, v in one.items()})
    return tokens, conf


@pytest.fixture
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    return torch.device("cuda:0")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(sample.CONFIDENCES))
@pytest.mark.parametrize("which", range(len(PARAMS)))
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_parameters(dev, dtype, which, kind):
    gen = torch.Generator().manual_seed(7 + which)
    for how in ("normal", "peaked", "ties"):
        run_rows(make((5, 2003), how, DTYPES[dtype], gen), torch.rand(5, generator=gen), PARAMS[which], kind, dev)


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2, 3, 4, 5, 9, 11])
@pytest.mark.parametrize("how", ["equal", "near", "zeros", "wide", "masked", "holes", "rising"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_values(dev, dtype, how, which):
    gen = torch.Generator().manual_seed(31 + which)
    for kind in sample.CONFIDENCES:
        run_rows(make((6, 4099), how, DTYPES[dtype], gen), torch.rand(6, generator=gen), PARAMS[which], kind, dev)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 63, 64, 65, 127, 511, 513, 1025, 4096, 32000, 50257, 126464, 152064, 262143, 262144])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_sizes(dev, dtype, vocab):
    gen = torch.Generator().manual_seed(vocab)
    for n, params in enumerate((PARAMS[0], PARAMS[1], PARAMS[5])):
        run_rows(make((3, vocab), ("normal", "peaked")[n % 2], DTYPES[dtype], gen), torch.rand(3, generator=gen), params, list(sample.CONFIDENCES)[n], dev)


@pytest.mark.gpu
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (5, 3), (64, 0), (7, 8)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_strides(dev, dtype, pad, offset):
    """Rows at any distance and address; what lies between and around them is not read."""
    gen = torch.Generator().manual_seed(pad + 100 * offset)
    rows, vocab = 7, 1237
    logits = make((rows, vocab), "normal", DTYPES[dtype], gen)
    buffer = torch.full((offset + rows * (vocab + pad) + 64,), INF, dtype=DTYPES[dtype], device=dev)
    view = torch.as_strided(buffer, (rows, vocab), (vocab + pad, 1), offset)
    view.copy_(logits)
    for params in (PARAMS[0], PARAMS[1], PARAMS[5]):
        run_rows(view, torch.rand(rows, generator=gen), params, "entropy", dev)
    one = view[:1].expand(4, vocab)  # a single row, over and over
    run_rows(one, torch.rand(4, generator=gen), PARAMS[1], "probability", dev)


@pytest.mark.gpu
@pytest.mark.parametrize("filters", [dict(top_p=0.9), dict(), dict(top_k=13), dict(min_p=0.01), dict(top_k=300, top_p=0.5, min_p=0.1)])
@pytest.mark.parametrize("vocab", [777, 20000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_ends_of_the_uniform_numbers(dev, dtype, vocab, filters):
    """The ends of u, and numbers that are none of it."""
    gen = torch.Generator().manual_seed(3)
    logits = make((8, vocab), "normal", DTYPES[dtype], gen)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -1.0, math.nan, 2.0 ** -149, 0.5])
    tokens, _ = sample.tokens(logits.to(dev), u.to(dev), temperature=1.0, **filters)
    tokens = tokens.cpu()
    for r in range(8):
        order, w, _ = ranked(logits[r].double().numpy(), 1.0, **{k: v if k == "top_k" else float(np.float32(v)) for k, v in filters.items()})
        last = order[int((w > 0).sum()) - 1]
        if r in (0, 4, 5, 6):
            assert tokens[r] == order[0]
        elif r in (2, 3):
            assert tokens[r] == last
        elif r == 1:  # up to 2^-24 short of the last weight
            assert order.tolist().index(int(tokens[r])) == min(int(np.searchsorted(np.cumsum(w), float(u[1]) * w.sum(), side="right")), int((w > 0).sum()) - 1)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [5, 256])
@pytest.mark.parametrize("how", ["equal", "near", "zeros"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_last_token_of_flat_rows(dev, dtype, how, rows):
    """Draws at the end of long rows whose weights are beyond 2^53 in units of 2^-44."""
    gen = torch.Generator().manual_seed(24)
    logits = make((5, 50257), how, DTYPES[dtype], gen)
    u = torch.tensor([1.0, 1.0 - 2.0 ** -24, INF, 2.0, 0.9999])
    for params in (dict(temperature=1.0), dict(temperature=2.0, top_k=30000), dict(temperature=1.0, top_p=0.9), dict(temperature=1.0, min_p=0.9)):
        tokens, _ = sample.tokens(logits.to(dev).repeat(rows // 5 + 1, 1)[:rows], u.to(dev).repeat(rows // 5 + 1)[:rows], **params)
        for r in range(5):
            order, w, _ = ranked(logits[r].double().numpy(), params["temperature"], **{k: v if k == "top_k" else float(np.float32(v)) for k, v in params.items() if k != "temperature"})
            place, last = int(np.flatnonzero(order == int(tokens[r]))[0]), int((w > 0).sum()) - 1
            if r in (0, 2, 3):
                assert place == last
            else:  # (weights are held to 2^-33 of themselves)
                assert 0 <= place <= last and abs(w[:place + 1].sum() - float(u[r]) * w.sum()) <= w[place] + 1e-9 * w.sum()
        assert (tokens.view(-1)[:5] == tokens[rows // 5 * 5 - 5:rows // 5 * 5]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_halves_to_the_last_bit(dev, dtype):
    # six equal tokens, u M = 3 exactly
    equal = torch.full((4, 6), 2.5, dtype=DTYPES[dtype], device=dev)
    tokens, conf = sample.tokens(equal, torch.tensor([0.0, 0.5, 0.5 - 2.0 ** -25, 1.0], device=dev), temperature=0.7)
    assert tokens.tolist() == [0, 3, 2, 5] and conf.tolist() == [float(np.float32(1 / 6))] * 4
    tokens, conf = sample.tokens(equal, torch.full((4,), 0.99, device=dev), temperature=0.7, top_p=0.5)
    assert tokens.tolist() == [2] * 4 and conf.tolist() == [float(np.float32(1 / 3))] * 4
    many = torch.zeros((2, 4096), dtype=DTYPES[dtype], device=dev)  # more of them than are sorted
    tokens, conf = sample.tokens(many, torch.tensor([0.5, 0.25], device=dev), temperature=1.0, top_p=0.5)
    assert tokens.tolist() == [1024, 512] and conf.tolist() == [1 / 2048] * 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_zeros_and_far_values_among_others(dev, dtype):
    """Zeros, tiny and huge logits last, first and in the middle of the ranks, where bf16 has no counts of its own for them."""
    gen = torch.Generator().manual_seed(21)
    rows = []
    for other in (torch.rand(700, generator=gen) + 0.1, -torch.rand(700, generator=gen) - 0.1, torch.randn(700, generator=gen)):
        for few in (torch.zeros(40), torch.full((40,), 1e-20), torch.full((40,), -3e-9), torch.full((1,), 300.0), torch.full((40,), -300.0),
                    torch.cat([torch.zeros(20), -torch.zeros(20)])):
            x = torch.cat([other, few, few.flip(0)[:5], torch.full((100 - len(few) - min(5, len(few)),), -INF)])
            rows.append(x[torch.randperm(len(x), generator=gen)])
    logits = torch.stack(rows).to(DTYPES[dtype])
    n = len(rows)
    for params in (dict(temperature=2.0), dict(temperature=30.0), dict(temperature=1.0, top_k=720), dict(temperature=5.0, top_p=0.97), dict(temperature=3.0, min_p=0.6),
                   dict(temperature=0.0), dict(temperature=200.0, top_k=710, min_p=0.3)):
        for u in (torch.rand(n, generator=gen), 1 - 2.0 ** -10 * torch.rand(n, generator=gen), 2.0 ** -10 * torch.rand(n, generator=gen)):
            for kind in sample.CONFIDENCES:
                run_rows(logits, u, params, kind, dev)


@pytest.mark.gpu
def test_more_rows_than_a_launch_takes(dev):
    """Rows beyond those of the first launch, with parameters a row."""
    rows = (1 << 23) + 700
    logits = torch.zeros((rows, 2), dtype=torch.float32, device=dev)
    logits[:, 1] = (torch.arange(rows, device=dev) % 3 - 1).float()
    temperature = (torch.arange(rows, device=dev) % 2).float()
    top_k = (torch.arange(rows, device=dev) % 5 == 0).int()
    tokens, conf = sample.tokens(logits, torch.full((rows,), 0.999999, device=dev), temperature=temperature, top_k=top_k)
    first = (logits[:, 1] > 0).int()
    last = torch.where((temperature > 0) & (top_k == 0), 1 - first, first)
    assert torch.equal(tokens, last)
    e = torch.exp(-logits[:, 1].double().abs())
    want = torch.where(top_k > 0, 1.0, torch.where(tokens == first, 1.0, e) / (1.0 + e))
    assert (conf.double() - want).abs().max() <= 2.0 ** -19


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_parameters_of_requests(dev, dtype):
    """Parameters by request, rows in any order of requests, rows of none."""
    gen = torch.Generator().manual_seed(11)
    rows, vocab, requests = 40, 5003, 9
    logits = make((rows, vocab), "peaked", DTYPES[dtype], gen)
    u = torch.rand(rows, generator=gen)
    each = dict(temperature=torch.tensor([0.0, 0.5, 1.0, 1.5, 0.7, -1.0, math.nan, 1.0, 0.9]), top_k=torch.tensor([0, 5, 0, 100, -3, 0, 0, 1, 4000], dtype=torch.int32),
                top_p=torch.tensor([1.0, 0.9, 0.3, 1.0, 2.0, 1.0, math.nan, 1.0, 0.99]), min_p=torch.tensor([0.0, 0.0, 0.1, 0.01, -1.0, 0.0, math.nan, 0.0, 0.0]))
    of = torch.randint(0, requests, (rows,), generator=gen, dtype=torch.int32)
    of[5], of[17] = -1, requests
    tokens, conf = sample.tokens(logits.to(dev), u.to(dev), **{k: v.to(dev) for k, v in each.items()}, params_of=of.to(dev), confidence="margin")
    plain = lambda v, off, ok: float(v) if ok(v) else off  # noqa: E731
    for r in range(rows):
        p = int(of[r])
        if not 0 <= p < requests:
            assert (int(tokens[r]), float(conf[r])) == (-1, 0.0)
            continue
        check(logits[r].double().numpy(), int(tokens[r]), float(conf[r]), float(u[r]), plain(each["temperature"][p], 0.0, lambda v: v > 0), "margin",
              max(0, int(each["top_k"][p])), plain(each["top_p"][p], 1.0, lambda v: v < 1), plain(each["min_p"][p], 0.0, lambda v: v > 0))
    # an entry a row, numbers beside it; and rows that are skipped without any array
    t = torch.rand(rows, generator=gen) + 0.3
    run_rows(logits, u, dict(temperature=t, top_k=30), "probability", dev)
    of = torch.where(torch.arange(rows) % 3 == 0, -1, 4).int()
    tokens, _ = sample.tokens(logits.to(dev), u.to(dev), temperature=0.0, params_of=of.to(dev))
    assert (tokens.cpu()[of < 0] == -1).all() and (tokens.cpu()[of >= 0] >= 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_forbidden_token(dev, dtype):
    gen = torch.Generator().manual_seed(5)
    for vocab in (1, 9, 1000, 4097):
        logits = make((4, vocab), "normal", DTYPES[dtype], gen)
        for forbid in sorted({0, vocab // 2, vocab - 1, int(logits[0].argmax())}):
            for params in (PARAMS[0], PARAMS[5]):
                tokens, _ = run_rows(logits, torch.rand(4, generator=gen), params, "probability", dev, forbid=forbid)
                assert (tokens != forbid).all()


@pytest.mark.gpu
def test_streams_outputs_and_graphs(dev):
    gen = torch.Generator().manual_seed(9)
    logits = make((33, 3001), "peaked", torch.bfloat16, gen).to(dev)
    u = torch.rand(33, generator=gen).to(dev)
    want = sample.tokens(logits, u, temperature=0.8, top_k=50, confidence="entropy")
    for _ in range(3):  # the same bits every time
        assert all(torch.equal(a, b) for a, b in zip(want, sample.tokens(logits, u, temperature=0.8, top_k=50, confidence="entropy")))
    out, conf = torch.full((33,), -7, dtype=torch.int32, device=dev), torch.zeros(33, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sample.tokens(logits, u, temperature=0.8, top_k=50, confidence="entropy", out=out, confidence_out=conf, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got[0] is out and all(torch.equal(a, b) for a, b in zip(want, got))
    # a captured step: tokens, then the rows that take them, on new numbers before each replay
    ids0 = torch.full((33,), 3001, dtype=torch.int32, device=dev)
    indptr = torch.tensor([0, 1, 1, 20, 33], dtype=torch.int32, device=dev)
    with torch.cuda.stream(side):
        sample.unmask(*sample.tokens(logits, u, temperature=0.8, top_k=50), ids0, indptr, mask_id=3001)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = sample.tokens(logits, u, temperature=0.8, top_k=50)
        h = sample.unmask(*g, ids0, indptr, mask_id=3001, count=2)
    for k in range(4):
        u.copy_(torch.rand(33, generator=gen))
        logits.copy_(make((33, 3001), ("peaked", "normal", "ties", "equal")[k], torch.bfloat16, gen))
        graph.replay()
        a = sample.tokens(logits, u, temperature=0.8, top_k=50)
        b = sample.unmask(*a, ids0, indptr, mask_id=3001, count=2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + b, g + h))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_next_to_zero(dev, dtype):
    """Logits so near 0 that their weights are that of 0, as the largest, among others and around the last that is kept."""
    gen = torch.Generator().manual_seed(22)
    for scale, rest in ((1e-20, -1.0), (1e-20, 1.0), (1e-30, 0.0), (1e-12, -40.0), (1e-38, 1e-12)):
        x = torch.full((6, 3001), rest) * (1 + torch.rand((6, 3001), generator=gen))
        x[:, ::7] = scale * torch.randn((6, 429), generator=gen)
        for params in (PARAMS[0], PARAMS[1], dict(temperature=0.9, top_k=200), dict(temperature=0.9, top_k=429), dict(temperature=30.0, top_p=0.1), dict(temperature=1e-15)):
            for kind in sample.CONFIDENCES:
                run_rows(x.to(DTYPES[dtype]), torch.rand(6, generator=gen), params, kind, dev)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(sample.CONFIDENCES))
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_powers_of_two_among_the_largest(dev, dtype, kind):
    """The largest logits on both sides of each power of two, where the sums of bf16's values begin anew."""
    gen = torch.Generator().manual_seed(25)
    for high in (256.0, 128.0, 64.0, 2.0, 0.5, 2.0 ** -10, -2.0 ** -10, -1.0, -64.0, -128.0):
        x = high * (1 + 0.03 * torch.rand((5, 1111), generator=gen))
        x[:, ::3] = high * (1 - 0.02 * torch.rand((5, 371), generator=gen))
        x[0, 5:] = high * 0.98
        x[1, 5:] = -300.0
        for params in (dict(temperature=0.0, top_k=2), dict(temperature=1.0, top_k=17), dict(temperature=1.0, min_p=1e-5), dict(temperature=0.5 * abs(high), top_p=0.6),
                       dict(temperature=3.0, top_k=134, min_p=0.006), dict(temperature=1.0)):
            run_rows(x.to(DTYPES[dtype]), torch.rand(5, generator=gen), params, kind, dev)


# rows that are split over work-groups (fewer than 256 of a long vocabulary), and rows of which a work-group takes a whole one
LONG = 20011


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2, 5, 9, 11])
@pytest.mark.parametrize("how", ["peaked", "ties", "equal", "near", "zeros", "wide", "masked", "holes", "rising"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_long_rows(dev, dtype, how, which):
    gen = torch.Generator().manual_seed(71 + which)
    for kind in sample.CONFIDENCES:
        run_rows(make((6, LONG), how, DTYPES[dtype], gen), torch.rand(6, generator=gen), PARAMS[which], kind, dev)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(sample.CONFIDENCES))
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_alone_and_among_many(dev, dtype, kind):
    """255, 256 and 300 rows against the definition, here and there, and each against itself in a call of few rows."""
    gen = torch.Generator().manual_seed(72)
    logits = make((300, LONG), "normal", DTYPES[dtype], gen)
    logits[7], logits[255] = -INF, math.nan
    logits[11, 100], logits[256, :9000] = INF, -INF
    u = torch.rand(300, generator=gen)
    temperature = torch.where(torch.arange(300) % 3 == 0, 0.0, torch.rand(300, generator=gen) + 0.3)
    top_k = torch.where(torch.arange(300) % 4 == 0, 0, torch.randint(1, 500, (300,), generator=gen)).int()
    there = logits.to(dev)
    at = torch.tensor([0, 3, 7, 11, 12, 100, 254, 255, 256, 299])
    for params in (dict(temperature=temperature, top_k=top_k), dict(temperature=0.0), dict(temperature=0.8, top_p=0.9)):
        of = lambda n: {k: v[n].to(dev) if torch.is_tensor(v) else v for k, v in params.items()}  # noqa: E731
        few, few_conf = run_rows(logits[at], u[at], {k: v[at] if torch.is_tensor(v) else v for k, v in params.items()}, kind, dev)
        for rows in (255, 256, 300):
            tokens, conf = sample.tokens(there[:rows], u[:rows].to(dev), confidence=kind, **of(slice(rows)))
            here = at < rows
            for r, token, c in zip(at[here].tolist(), tokens.cpu()[at[here]], conf.cpu()[at[here]]):
                one = {k: (v[r].item() if torch.is_tensor(v) else float(np.float32(v))) for k, v in params.items()}
                check(logits[r].double().numpy(), int(token), float(c), float(u[r]), kind=kind, **one)
            # (weights of bf16 rows are summed alike; places of others are whole numbers)
            assert torch.equal(tokens[at[here].to(dev)], few[here.to(dev)])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_graphs_of_long_rows(dev, dtype):
    """Two captured calls with parts of rows, replayed in turn and with eager calls between them."""
    gen = torch.Generator().manual_seed(73)
    x, y = (make((5, LONG), how, DTYPES[dtype], gen).to(dev) for how in ("peaked", "normal"))
    u = torch.rand(5, generator=gen).to(dev)
    greedy, drawn = dict(temperature=0.0, confidence="entropy"), dict(temperature=0.9, top_p=0.95, confidence="margin")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sample.tokens(x, u, **greedy)
        sample.tokens(y, u, **drawn)
    torch.cuda.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        a = sample.tokens(x, u, **greedy)
    with torch.cuda.graph(two):
        b = sample.tokens(y, u, **drawn)
    for k in range(5):
        u.copy_(torch.rand(5, generator=gen))
        x.copy_(make((5, LONG), ("normal", "ties", "masked", "holes", "peaked")[k], DTYPES[dtype], gen))
        y.copy_(make((5, LONG), ("near", "masked", "peaked", "equal", "holes")[k], DTYPES[dtype], gen))
        one.replay()
        two.replay()
        want = sample.tokens(x, u, **greedy) + sample.tokens(y, u, **drawn)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a + b, want))


@pytest.mark.gpu
def test_rows_past_32_bits(dev):
    """Rows whose offsets in elements and bytes do not fit in 32 bits."""
    stride = (1 << 31) + 13
    gen = torch.Generator().manual_seed(74)
    for vocab in (LONG, 999):
        buffer = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device=dev)
        view = torch.as_strided(buffer, (3, vocab), (stride, 1), 0)
        view.copy_(make((3, vocab), "normal", torch.bfloat16, gen))
        for params in (PARAMS[0], PARAMS[5]):
            run_rows(view, torch.rand(3, generator=gen), params, "probability", dev)


# ------------------------------------------------------------------ far tails
def tails(vocab, T, others):
    """Rows whose last tokens of any weight are some tens of powers of two under the largest, in any dtype, and none within 0.2 of
    the 64th. All others have no weight: they are masked, or 69 powers of two under the largest."""
    fixed = [[30.0] + [-10.0] * 5,                                  # 2^-57.7
             [30.0, 29.0, 29.0, 3.0] + [-8.0] * 700 + [-12.0] * 3,  # 2^-54.8, more equal ones than are sorted, 2^-60.6
             [30.0, 12.0] + [-13.0] * 600,                          # 2^-62.0
             [40.0, 39.0] + [0.0, -0.0] * 30,                       # 2^-57.7
             [42.0, 7.0, 0.0, 0.0, -0.5, -0.5, -2.0],               # 2^-60.6, -61.3, -63.5
             [300.0, 290.0, 258.0, 258.0, 268.0],                   # 2^-60.6, beyond what bf16 counts
             [-2.0] * 9 + [-40.0] * 2 + [-45.0],                    # 2^-54.8, -62.0
             [20.0] * 40 + [-4.5, -5.0, -20.0]]                     # 2^-35.3, -36.1, -57.7
    gen = torch.Generator().manual_seed(vocab)
    x = torch.empty((len(fixed), vocab))
    for r, values in enumerate(fixed):
        x[r] = -INF if others == "masked" else (values[0] - 48.0) * T
        x[r, torch.randperm(vocab, generator=gen)[:len(values)]] = torch.tensor(values) * T
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("others", ["masked", "weightless"])
@pytest.mark.parametrize("rows,vocab", [(8, 1500), (8, 20011), (264, 20011)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_last_token_of_any_weight(dev, dtype, rows, vocab, others):
    """u from 1 on takes the last kept token of any weight (2^-64 of the largest at least), also where it is under what sums
    hold. Confidences: one rounding to 32 bits, and 2^-33 of the weight and of the sum."""
    for T in (1.0, 0.5, 4.0):
        x = tails(vocab, T, others).to(DTYPES[dtype])
        n = x.shape[0]
        u = torch.tensor([1.0, 2.0, INF, 1.0, 1.0, 3.0, 1.0, 1.0])
        for params in (dict(), dict(top_k=vocab - 1), dict(top_k=300), dict(top_k=6), dict(top_k=2), dict(min_p=1e-18), dict(min_p=1e-30), dict(top_p=1.0 - 2.0 ** -24),
                       dict(top_k=700, min_p=1e-17, top_p=0.99)):
            tokens, conf = sample.tokens(x.to(dev).repeat(rows // n, 1), u.to(dev).repeat(rows // n), temperature=T, **params)
            tokens, conf = tokens.cpu().view(-1, n), conf.cpu().view(-1, n)
            assert (tokens == tokens[0]).all() and (conf == conf[0]).all()
            for r in range(n):
                order, w, z = ranked(x[r].double().numpy(), T, **{k: v if k == "top_k" else float(np.float32(v)) for k, v in params.items()})
                bits = z / math.log(2.0)
                assert not ((w > 0) & (abs(bits + 64) < 0.2)).any()
                last = int(((w > 0) & (bits > -64)).sum()) - 1
                assert int(tokens[0, r]) == order[last], (T, params, r)
                ref = w[last] / w.sum()
                assert abs(float(conf[0, r]) - ref) <= (2.0 ** -24 * (1 + 2.0 ** -6) + 2.0 ** -32) * ref, (T, params, r)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 260])
def test_lowest_numbers_under_large_temperatures(dev, rows):
    """Logits of the type's lowest value have weight, and min-p keeps them, where the temperature is that large."""
    gen = torch.Generator().manual_seed(26)
    for dtype in DTYPES.values():
        x = torch.randn((rows, 20011), generator=gen).to(dtype)
        x[:, ::3] = torch.finfo(dtype).min
        x[0, 1:] = torch.finfo(dtype).min
        x[1, 7] = torch.finfo(dtype).max
        u = torch.rand(rows, generator=gen)
        u[2:4] = torch.tensor([1.0, 1.0 - 2.0 ** -24])
        for T in (INF, 1e38, 3e38):
            for params in (dict(min_p=0.5), dict(min_p=0.02), dict(min_p=0.02, top_k=15000), dict(top_p=0.9, min_p=1e-4), dict()):
                for kind in sample.CONFIDENCES:
                    there, of = x.to(dev), dict(temperature=T, **params)
                    tokens, conf = sample.tokens(there, u.to(dev), confidence=kind, **of)
                    for r in range(6):
                        check(x[r].double().numpy(), int(tokens[r]), float(conf[r]), float(u[r]), kind=kind, **{k: v if k == "top_k" else float(np.float32(v)) for k, v in of.items()})


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_entropies_in_any_order(dev, dtype):
    """The entropy of what is kept is the same to the last bit every time, in few and in many rows, and for every order of the
    row's tokens: which thread adds what changes nothing."""
    gen = torch.Generator().manual_seed(27)
    for how in ("normal", "peaked", "rising", "near", "holes"):
        x = make((9, LONG), how, DTYPES[dtype], gen).to(dev)
        u = torch.rand(9, generator=gen).to(dev)
        for params in (dict(temperature=1.0), dict(temperature=0.7, top_k=2000), dict(temperature=1.2, top_p=0.9), dict(temperature=0.0, min_p=1e-4)):
            one = lambda t, n=1: sample.tokens(t.repeat(n, 1), u.repeat(n), confidence="entropy", **params)[1]  # noqa: E731
            want = one(x)
            for _ in range(5):
                assert torch.equal(one(x), want)
                assert torch.equal(one(x[:, torch.randperm(LONG, generator=gen).to(dev)]), want)
            assert torch.equal(one(x, 30).view(30, 9), want.expand(30, 9))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(sample.CONFIDENCES))
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_confidences_in_few_and_many_rows(dev, dtype, kind):
    """A row's confidence is its own, to the last bit. That of the first token of everything in fp16 and fp32 rows is off by 2^-19
    of the sum at most (entropy: times 2 + log(vocab)), in few rows and in many."""
    gen = torch.Generator().manual_seed(28)
    for how in ("normal", "peaked", "wide", "holes", "zeros"):
        x = make((6, LONG), how, DTYPES[dtype], gen).to(dev)
        u = torch.rand(6, generator=gen).to(dev)
        for params in (dict(temperature=0.8), dict(temperature=1.0, top_k=40), dict(temperature=1.3, top_p=0.9), dict(temperature=0.0, min_p=0.01), dict(temperature=0.0)):
            few, many = (sample.tokens(x.repeat(n, 1), u.repeat(n), confidence=kind, **params) for n in (1, 50))
            assert torch.equal(many[0].view(50, 6), few[0].expand(50, 6))
            if len(params) > 1 or params["temperature"] > 0 or dtype == "bf16":
                assert torch.equal(many[1].view(50, 6), few[1].expand(50, 6))
            else:
                bar = 2 * 2.0 ** -19 * (2 + math.log(LONG) if kind == "entropy" else few[1].abs().double() + (1.0 if kind == "margin" else 0.0))
                assert ((many[1].view(50, 6).double() - few[1].double()).abs() <= bar).all()


def test_exact_sums(tmp_path):
    """The sum that these entropies take, on the host: the same bits in every order, of up to 2^18 numbers, each added to 2^-84."""
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(os.path.dirname(os.path.abspath(__file__)), "sanitize", "exact_sum_driver.cpp"), "-o", exe], check=True)
    rng = np.random.default_rng(6)
    cases = [rng.random(1000), 34 * 2.0 ** -rng.uniform(0, 66, 5000), np.full(1 << 18, 34.0), np.full(1 << 18, np.nextafter(64.0, 0.0)), 2.0 ** -rng.uniform(30, 90, 3000),
             np.array([0.0, 2.0 ** -38, 1.5 * 2.0 ** -38, 2.0 ** -39, 33.999]), np.zeros(0)]
    for x in cases:
        text, orders = "", 3 if len(x) < 10000 else 1
        for k in range(orders):
            text += " ".join([str(len(x))] + [float(v).hex() for v in (rng.permutation(x) if k else x)]) + "\n"
        out = [line.split() for line in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()]
        assert len(out) == orders and all(o == out[0] for o in out)
        want = math.fsum(x)
        assert abs(float.fromhex(out[0][2]) - want) <= len(x) * 2.0 ** -84 + 2.0 ** -52 * want
    # a sum of doubles does hang on the order
    x = cases[1]
    assert len({float(np.cumsum(rng.permutation(x))[-1]) for _ in range(20)}) > 1


def test_workspace():
    """Parts of rows need memory; too little of it, or at an odd address, is refused before any HIP call."""
    lib, bytes_of = _lib.lib, _lib.lib.sangam_sample_workspace_bytes
    assert bytes_of(4, 100, 0) == bytes_of(256, LONG, 0) == bytes_of(0, LONG, 0) == bytes_of(-1, LONG, 0) == bytes_of(4, LONG, 7) == bytes_of(4, 0, 0) == 0
    assert bytes_of(4, 2 ** 18 + 1, 0) == bytes_of(2 ** 31, LONG, 0) == 0
    for dtype in range(3):
        need = bytes_of(4, LONG, dtype)
        assert need > 0
        desc = c_desc(vocab=LONG, row_stride=LONG, dtype=dtype)
        assert lib.sangam_sample_tokens(ctypes.byref(desc), 4096, 4096, None, need, None) == -5
        assert lib.sangam_sample_tokens(ctypes.byref(desc), 4096, 4096, 4096, need - 1, None) == -5
        assert lib.sangam_sample_tokens(ctypes.byref(desc), 4096, 4096, 4096 + 128, need, None) == -6


@pytest.mark.gpu
def test_no_rows(dev):
    tokens, conf = sample.tokens(torch.empty((0, 50), device=dev), torch.empty(0, device=dev))
    assert tokens.shape == conf.shape == (0,)


def test_definition():
    """The oracle's own words on a row that can be followed by hand."""
    x = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    order, w, _ = ranked(x, 1.0)
    assert order.tolist() == [1, 2, 3, 0, 4]
    np.testing.assert_allclose(w / w.sum(), [0.4, 0.2, 0.2, 0.1, 0.1], rtol=1e-12)
    assert (ranked(x, 1.0, top_k=3)[1] > 0).tolist() == [True, True, True, False, False]
    assert (ranked(x, 1.0, top_p=0.55)[1] > 0).tolist() == [True, True, False, False, False]
    assert (ranked(x, 1.0, top_k=2, top_p=0.65)[1] > 0).tolist() == [True, False, False, False, False]
    assert (ranked(x, 1.0, min_p=0.45)[1] > 0).tolist() == [True, True, True, False, False]
    assert (ranked(x, 1.0, top_p=0.0)[1] > 0).tolist() == [True, False, False, False, False]
    assert ranked([-INF, math.nan], 1.0) is None
    assert ranked([1.0, INF, INF, -INF], 1.0)[1].tolist() == [1.0, 1.0, 0.0, 0.0]


# ------------------------------------------------------------------ refusals
def c_desc(**kw):
    d = _lib.SampleDesc(4096, 4, 100, 100, 0, 4096, None, 0, None, None, None, None, 1.0, 0, 1.0, 0.0, 0, -1)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("status,kw", [
    (-2, dict(dtype=3)), (-2, dict(dtype=-1)), (-1, dict(rows=-1)), (-1, dict(rows=2 ** 31)), (-1, dict(vocab=0)), (-1, dict(vocab=2 ** 18 + 1)),
    (-1, dict(confidence=3)), (-1, dict(confidence=-1)), (-1, dict(forbid=-2)), (-1, dict(forbid=100)), (-1, dict(temperature=-0.5)),
    (-1, dict(temperature=math.nan)), (-1, dict(top_k=-1)), (-1, dict(top_p=1.5)), (-1, dict(top_p=-0.1)), (-1, dict(top_p=math.nan)), (-1, dict(min_p=2.0)),
    (-1, dict(min_p=math.nan)), (-1, dict(num_params=-1)), (-1, dict(temperatures=4096, num_params=3)), (-1, dict(logits=None)), (-1, dict(u=None)),
    (-1, dict(row_stride=-1)), (-1, dict(row_stride=2 ** 40 + 1)), (-6, dict(logits=4097)), (-6, dict(dtype=2, logits=4098)), (-6, dict(u=4098)),
    (-6, dict(params_of=4097, num_params=4)), (-6, dict(top_ks=4099, num_params=4))])
def test_c_refusals(status, kw):
    """Fake addresses: every check fails before any HIP call."""
    assert _lib.lib.sangam_sample_tokens(ctypes.byref(c_desc(**kw)), 4096, 4096, None, 0, None) == status
    assert len(_lib.lib.sangam_last_error()) > 0


def test_c_outputs_refused():
    lib = _lib.lib
    assert lib.sangam_sample_tokens(None, 4096, 4096, None, 0, None) == -1
    assert lib.sangam_sample_tokens(ctypes.byref(c_desc()), None, 4096, None, 0, None) == -1
    assert lib.sangam_sample_tokens(ctypes.byref(c_desc()), 4097, 4096, None, 0, None) == -6
    assert lib.sangam_sample_tokens(ctypes.byref(c_desc()), 4096, 4098, None, 0, None) == -6
    assert lib.sangam_sample_tokens(ctypes.byref(c_desc(rows=0, logits=None, u=None)), None, None, None, 0, None) == 0


def test_python_refusals():
    x, u = torch.zeros((4, 10)), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        sample.tokens(x, u)
    with pytest.raises(TypeError):
        sample.tokens(x.double(), u)
    with pytest.raises(TypeError):
        sample.tokens(x[0], u)
    with pytest.raises(ValueError, match="confidence"):
        sample.tokens(x, u, confidence="mean")


@pytest.mark.gpu
def test_python_refusals_on_device(dev):
    x, u = torch.zeros((4, 10), device=dev), torch.zeros(4, device=dev)
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    for error, kw in [(ValueError, dict(temperature=-1.0)), (ValueError, dict(temperature=math.nan)), (ValueError, dict(top_k=-1)), (ValueError, dict(top_p=1.01)),
                      (ValueError, dict(min_p=-0.5)), (ValueError, dict(forbid=10)), (ValueError, dict(forbid=-2)), (TypeError, dict(temperature=ints(4))),
                      (ValueError, dict(temperature=u[:3])), (TypeError, dict(top_k=u)), (ValueError, dict(top_k=ints(5))), (ValueError, dict(params_of=ints(3))),
                      (TypeError, dict(params_of=u)), (ValueError, dict(params_of=ints(4), temperature=u[:2], top_k=ints(3))), (ValueError, dict(top_p=u.cpu())),
                      (TypeError, dict(out=u)), (ValueError, dict(out=ints(3))), (ValueError, dict(confidence_out=torch.zeros(8, device=dev)[::2]))]:
        with pytest.raises(error):
            sample.tokens(x, u, **kw)
    with pytest.raises(ValueError):
        sample.tokens(x, u[:3])
    with pytest.raises(ValueError):
        sample.tokens(x.t(), torch.zeros(10, device=dev))
    with pytest.raises(ValueError):
        sample.tokens(torch.zeros((1, 2 ** 18 + 1), device=dev), u[:1])
