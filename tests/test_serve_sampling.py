"""The serving loop with its block table on the device and with sampling
(paper_2607_04206_amd/serve.py): page lists, positions and slots of every batch
against the host's, tokens and confidences against their definition, the ids of
the pool step by step until every response is resolved; quantised and rotated as
a worker runs them."""
import math

import numpy as np
import pytest
import torch

import workloads
from paper_2607_04206_amd import sample, tables
from paper_2607_04206_amd.serve import PAGE, ServingLoop
from tests.test_sample import check, ranked
from tests.test_unmask import definition


def test_arguments():
    reqs = workloads.serving_trace(0, 10, 0.4, median=100)
    make = lambda **kw: ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=None, sampling=kw)  # noqa: E731
    for bad in (dict(vocab=0), dict(vocab=1 << 18), dict(vocab=100, count=0), dict(vocab=100, heat=1.0)):
        with pytest.raises(ValueError):
            make(**bad)
    loop = make(vocab=100, temperature=0.5, confidence="margin")
    loop.run(200)  # the host alone: the trace's steps
    assert all(s.phase == "done" for s in loop.reqs)


@pytest.mark.gpu
def test_block_table_follows_the_pool():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    reqs = workloads.serving_trace(5, 60, 0.8, median=120)
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=2048, device=torch.device("cuda:0"), rotary={})
    batches = 0
    for t in range(600):
        if not loop.busy():
            break
        rec = loop.step(t, timed=False, capture=True)
        if rec is None:
            continue
        c = rec.captured
        b = c["tables"]
        assert np.array_equal(b.page_ids.cpu().numpy(), c["page_ids"]) and np.array_equal(b.page_indptr.cpu().numpy(), c["page_indptr"])
        n = np.diff(c["q_indptr"])
        positions = np.concatenate([o + np.arange(k) for o, k in zip(c["q_offset"], n)])
        items = np.repeat(np.arange(len(n)), n)
        page = c["page_ids"][c["page_indptr"][items] + positions // PAGE].astype(np.int64)
        assert np.array_equal(b.positions.cpu().numpy(), positions) and np.array_equal(b.items.cpu().numpy(), items)
        assert np.array_equal(b.slots.cpu().numpy(), page * PAGE + positions % PAGE)
        batches += 1
    assert batches > 50 and all(s.phase == "done" for s in loop.reqs)
    assert loop.pool.free == loop.pool.num_pages


@pytest.mark.gpu
@pytest.mark.parametrize("how,threshold,loop_kw", [
    (dict(), 0.9, dict()), (dict(temperature=0.8, top_p=0.95), 0.5, dict(kv_format="e4m3", rotary={})),
    (dict(temperature=1.0, top_k=50, confidence="margin"), math.inf, dict()), (dict(confidence="entropy"), -2.0, dict(rotary={}))])
def test_sampling(how, threshold, loop_kw):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    reqs = workloads.serving_trace(7, 12, 0.5, median=100, resp=64)
    vocab = 1999
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=torch.device("cuda:0"), sampling=dict(vocab=vocab, count=3, threshold=threshold, **how), **loop_kw)
    params = {"temperature": 0.0, "top_k": 0, "top_p": 1.0, **how}
    kind = params.pop("confidence", "probability")
    steps = 0
    for t in range(2000):
        if not loop.busy():
            break
        before = loop.ids.cpu().numpy()
        rec = loop.step(t, timed=False, capture=True)
        if rec is None:
            continue
        nd, c = rec.decodes, rec.captured
        slots = c["tables"].slots.cpu().numpy()
        after = loop.ids.cpu().numpy()
        expect = before.copy()
        for k in range(nd, len(c["kv_len"])):  # prefills: only fresh ones mask their response
            rid = rec.batch[k][0]
            state = next(s for s in loop.reqs if s.req.rid == rid)
            if state.block == 0:
                expect[slots[c["q_indptr"][k] + state.req.prompt:c["q_indptr"][k + 1]]] = vocab
        if nd:
            rows = 32 * nd
            tokens, confidence, out = (x.cpu().numpy() for x in loop.sampled)
            if steps % 5 == 0 and params["temperature"] == 0:
                for r in range(0, rows, 7):
                    check(loop.logits[r].double().cpu().numpy(), int(tokens[r]), float(confidence[r]), 0.0, params["temperature"], kind, params["top_k"],
                          float(np.float32(params["top_p"])), forbid=vocab)
            assert (tokens >= 0).all() and (tokens < vocab).all()
            want, left = definition(tokens, confidence, expect[slots[:rows]], np.arange(0, rows + 1, 32), vocab, [3] * nd, [np.float32(threshold)] * nd)
            assert np.array_equal(out, want) and rec.left == left.tolist()
            expect[slots[:rows]] = want
            steps += 1
        assert np.array_equal(after, expect), f"iteration {t}"
    assert steps > 5 and all(s.phase == "done" for s in loop.reqs) and loop.pool.free == loop.pool.num_pages


@pytest.mark.gpu
@pytest.mark.parametrize("rotary", [None, {}])
def test_a_loop_that_reads_no_slots_makes_none(monkeypatch, rotary):
    """Without sampling the host's page list and positions are sent, and no table kernel runs, until a step is captured: then the
    block table has followed every request that came or went before."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    reqs = workloads.serving_trace(9, 40, 0.8, median=120)
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=2048, device=torch.device("cuda:0"), rotary=rotary)

    def unread(*args, **kw):
        raise AssertionError("a table that nothing reads")

    checked = gone = 0
    for t in range(600):
        if not loop.busy():
            break
        capture = t % 7 == 6
        with monkeypatch.context() as m:
            if not capture:
                m.setattr(tables, "resize", unread)
                m.setattr(tables, "build", unread)
            rec = loop.step(t, timed=False, capture=capture)
        if rec is None or not capture:
            continue
        c = rec.captured
        n = np.diff(c["q_indptr"])
        positions = np.concatenate([o + np.arange(k) for o, k in zip(c["q_offset"], n)])
        b = c["tables"]
        assert np.array_equal(b.page_ids.cpu().numpy(), c["page_ids"]) and np.array_equal(b.positions.cpu().numpy(), positions)
        assert np.array_equal(loop._positions(), positions)
        checked += 1
        gone = sum(s.phase == "done" for s in loop.reqs)
    assert checked > 10 and gone > 5 and all(s.phase == "done" for s in loop.reqs)


@pytest.mark.gpu
@pytest.mark.parametrize("sampling", [None, dict(vocab=999)])
def test_a_table_without_pages_is_noticed(monkeypatch, sampling):
    """A block table that no longer follows the host's pool ends the run, at the next look at the device's numbers."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    resize, calls = tables.resize, []

    def short(*args, **kw):  # the fourth call says that a request found none (all do: the pages are right)
        calls.append(resize(*args, **kw))
        if len(calls) == 4:
            calls[-1].fill_(1)
        return calls[-1]

    monkeypatch.setattr(tables, "resize", short)
    reqs = workloads.serving_trace(7, 12, 0.5, median=100, resp=64)
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=torch.device("cuda:0"), sampling=sampling)
    if sampling is None:  # (captured steps alone read the table then)
        for t in range(30):
            loop.step(t, timed=False, capture=True)
    with pytest.raises(RuntimeError, match="free pages"):
        loop.run(2000, timed=False)
    assert len(calls) >= 4


@pytest.mark.gpu
@pytest.mark.parametrize("how", [dict(temperature=0.8, top_p=0.6), dict(temperature=1.5, top_k=3, confidence="margin"), dict(temperature=2.0, min_p=0.02, confidence="entropy"),
                                 dict(temperature=3.0)])
def test_drawn_tokens(monkeypatch, how):
    """Tokens and confidences of drawn rows against their definition, from the uniform numbers that the loop gave. The parameters
    of the hotter ones matter: of some rows the definition without them takes another token."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    calls, tokens_of = [], sample.tokens

    def kept(logits, u, **kw):
        got = tokens_of(logits, u, **kw)
        calls.append((logits.double().cpu().numpy(), u.tolist(), got[0].tolist(), got[1].tolist()))
        return got

    monkeypatch.setattr(sample, "tokens", kept)
    reqs = workloads.serving_trace(7, 6, 0.5, median=100, resp=64)
    vocab = 1999
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=torch.device("cuda:0"), sampling=dict(vocab=vocab, count=4, **how))
    loop.run(2000, timed=False)
    kind = how.get("confidence", "probability")
    params = {k: v if k == "top_k" else float(np.float32(v)) for k, v in how.items() if k != "confidence"}
    others = 0
    for logits, u, tokens, confidence in calls[::max(1, len(calls) // 6)]:
        for r in range(0, len(u), 5):
            check(logits[r], tokens[r], confidence[r], u[r], kind=kind, forbid=vocab, **params)
            order, w, _ = ranked(np.where(np.arange(vocab + 1) == vocab, -math.inf, logits[r]), 1.0)
            others += int(tokens[r]) != int(order[min(int(np.searchsorted(np.cumsum(w), u[r] * w.sum(), side="right")), vocab - 1)])
    assert len(calls) > 1 and (others > 0 or how["temperature"] < 1) and all(s.phase == "done" for s in loop.reqs)
