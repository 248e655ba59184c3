"""The serving loop over a quantised KV cache and with rotary positions
(paper_2607_04206_amd/serve.py): rotation, the attention call with its quantised
write-back and its reads of what earlier iterations wrote, page after page of
reuse, as a worker runs them one behind the other."""
import numpy as np
import pytest
import torch

import workloads
from oracle import mx
from paper_2607_04206_amd import kv, kvq
from paper_2607_04206_amd.serve import ServingLoop
from tests.test_rope import rotated
from tests.test_serve import check_iteration


def test_arguments():
    reqs = workloads.serving_trace(0, 10, 0.4, median=100)
    make = lambda **kw: ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=None, **kw)  # noqa: E731
    with pytest.raises(ValueError):
        make(kv_format="e5m2")
    loop = make(kv_format="e2m1", rotary=dict(rot_dim=32, scaling="linear", factor=2.0))
    assert loop.rope.rot_dim == 32 and make(rotary={}).rope.rot_dim == 64
    loop.run(200)  # plans every batch, as without them
    assert all(s.phase == "done" for s in loop.reqs)


@pytest.mark.gpu
@pytest.mark.parametrize("kv_format,rotary", [("e4m3", None), ("e2m1", dict(interleaved=True)), ("e4m3", dict(rot_dim=32)),
                                              (None, dict(scaling="yarn", factor=4.0, original_len=256.0))])
def test_serving_loop(kv_format, rotary):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    dev = torch.device("cuda:0")
    reqs = workloads.serving_trace(3, 30, 0.5, median=150)
    loop = ServingLoop(reqs, hq=8, hkv=2, d=64, tau=1024, device=dev, kv_format=kv_format, rotary=rotary)
    assert (loop.cache is None) == (kv_format is None)
    checked, expected = 0, None
    for t in range(400):
        if not loop.busy():
            break
        rec = loop.step(t, timed=t % 7 == 0, capture=True)
        if rec is None:
            continue
        c = rec.captured
        pi = c["page_indptr"]
        # the pages that the last iteration left are those that this one finds
        if expected is not None:
            for page, k, v in zip(c["page_ids"], c["k_pages"].float().cpu(), c["v_pages"].float().cpu()):
                if int(page) in expected:
                    for got, (want, known) in zip((k, v), expected[int(page)]):
                        assert torch.equal(got[:, known], want[:, known]), f"iteration {t}, page {page}"
        expected = {}
        for i in range(len(c["kv_len"])):
            pos = np.arange(int(c["q_indptr"][i + 1] - c["q_indptr"][i])) + int(c["q_offset"][i])
            new = [c[n][int(c["q_indptr"][i]):int(c["q_indptr"][i + 1])].double().cpu().numpy() for n in ("k_new", "v_new")]
            if kv_format:
                new = [mx.values(*mx.quantise(x, kv_format), kv_format) for x in new]
            for n, page in enumerate(c["page_ids"][pi[i]:pi[i + 1]]):
                known = torch.arange(16 * n, 16 * n + 16) < int(c["kv_len"][i])
                entry = []
                for pages, x in zip((c["k_pages"], c["v_pages"]), new):
                    was = pages[pi[i] + n].float().cpu()
                    here = (pos // 16) == n
                    was[:, pos[here] % 16] = torch.from_numpy(x[here]).float().transpose(0, 1)
                    entry.append((was, known))
                expected[int(page)] = entry
        if rotary is not None and t < 3:
            rows = c["q"].shape[0]
            at = np.concatenate([np.arange(n) + o for n, o in zip(np.diff(c["q_indptr"]), c["q_offset"])])
            scale = {k: v for k, v in rotary.items() if k not in ("rot_dim", "interleaved")}
            for got, x in ((c["q"], loop.q[:rows]), (c["k_new"], loop.k_new[:rows])):
                want, bar = rotated(x.double().cpu().numpy(), at, rotary.get("rot_dim", 64), rotary.get("interleaved", False), **scale)
                assert (np.abs(got.double().cpu().numpy() - want) <= bar + 2.0 ** -8 * (np.abs(want) + bar)).all()
        if rec.decodes and rec.prefills and checked < 3:
            print(f"[case] serving loop {kv_format} {rotary} iteration {t}: {rec.decodes} decodes, {rec.prefills} prefills", flush=True)
            check_iteration(c)
            checked += 1
    assert checked == 3 and all(s.phase == "done" for s in loop.reqs)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_prefill_hand_off_decode(fmt):
    """A prefill worker's call fills quantised pages, the rows go through a
    hand-off into another pool under another page table, and a block decode
    there gives the bits that it gives on the first pool."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from tests.test_kvq import plan_of, quant_inputs, quantised
    dev = torch.device("cuda:0")
    pre = workloads.make_workload("pre", 1, hq=8, hkv=2, d=128, decodes=[], prefills=[333, 90, 700])
    t, cache, _, _ = quant_inputs(pre, dev, fmt)
    kvq.forward(plan_of(pre, dev), t["q"], t["k_new"], t["v_new"], cache, t["page_ids"])
    table = dict(kv_len=pre.kv_len, page_indptr=pre.page_indptr, num_kv_heads=2, head_dim=128, num_pool_pages=pre.num_pool_pages, device=dev)
    other_ids = np.random.default_rng(9).permutation(pre.num_pool_pages)[:len(pre.page_ids)].astype(np.int32)
    other = kvq.empty_cache(pre.num_pool_pages, 2, 128, format=fmt, device=dev)
    kvq.kv_import(kv.plan(page_ids=other_ids, **table), *kvq.kv_export(kv.plan(page_ids=pre.page_ids, **table), cache), other)
    dec = workloads.make_workload("dec", 2, hq=8, hkv=2, d=128, decodes=[(300, 333), (0, 90), (640, 700)], prefills=[])
    outs = []
    for ids, c in ((pre.page_ids, cache), (other_ids, other)):
        dec.page_ids, dec.num_pool_pages = ids, pre.num_pool_pages
        outs.append(kvq.forward(plan_of(dec, dev), dec.packed_q(dev), dec.packed_k_new(dev), dec.packed_v_new(dev), c,
                                torch.from_numpy(ids).to(dev)))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0].view(torch.int16), outs[1][0].view(torch.int16)) and torch.equal(outs[0][1], outs[1][1])
    assert torch.isfinite(outs[0][0].float()).all()
