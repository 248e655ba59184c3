"""Prefill blocks of a mixed launch over a quantised cache (xcd_order.h), listed
on the CPU: each block's tile once, and the blocks of a round that share an XCD
are of few heads, also where the planner has ordered the tiles already. (GPU)
Such a launch against the oracle."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import workloads
from tests import test_plan
from tests.test_kvq import FMTS, dev, plan_of, run_case  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    exe = str(tmp_path_factory.mktemp("xcd") / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(HERE, "sanitize", "xcd_order_driver.cpp"), "-o", exe], check=True)

    def listed(tiles, rows, cus):
        r = subprocess.run([exe], input=f"{tiles} {rows} {cus}", capture_output=True, text=True, timeout=120, check=True)
        chunk, *out = (int(x) for x in r.stdout.split())
        return chunk, np.asarray(out)
    return listed


@pytest.mark.parametrize("rows", [128, 256])
def test_every_block_once(blocks, rows):
    rng = np.random.default_rng(0)
    for tiles, cus in [(1, 256), (7, 256), (255, 256), (256, 8), (257, 8), (2048, 256), (4099, 256), (1000, 1), (900, 15), (3000, 304)] + \
            [(int(np.exp(rng.uniform(0, 9))), int(rng.choice([1, 7, 8, 64, 256]))) for _ in range(40)]:
        chunk, got = blocks(tiles, rows, cus)
        slots = 8 * max(1, cus // 8) * (1 if rows == 256 else 2)
        assert chunk == (slots if tiles >= 8 * slots else 0)
        want = np.arange(2 * tiles) if rows == 256 else 2 * np.arange(tiles)
        assert np.array_equal(np.sort(got), want), (tiles, cus)


@pytest.mark.parametrize("cus", [1 << 28, 1 << 30, 2 ** 31 - 1])
def test_plans_for_any_number_of_cus(blocks, cus):
    for rows, wide in ((128, 1), (256, 2)):
        chunk, got = blocks(70, rows, cus)
        assert chunk == 0 and np.array_equal(np.sort(got), np.arange(70 * wide) * (2 // wide))
    wl = workloads.make_workload("cus", 1, hq=4, hkv=4, d=64, decodes=[(30, 100)], prefills=[300, 70])
    few, many = plan_of(wl), plan_of(wl, num_cus=cus)
    assert few.info.num_prefill_tiles == many.info.num_prefill_tiles


# a short launch, long ones that the planner orders (of 256 and 128 rows a tile)
@pytest.mark.parametrize("prefills,d,ordered,heads", [([1819, 1201], 128, False, 4.5), ([900] * 16, 128, True, 8.8),
                                                      ([3400] * 5, 128, True, 2.8), ([3400] * 5, 64, True, 2.2), ([900] * 16, 64, True, 8.8)])
def test_an_xcd_has_few_heads(blocks, prefills, d, ordered, heads):
    wl = workloads.make_workload("xcd", 1, hq=32, hkv=32, d=d, decodes=[(300, 1000)] * 64, prefills=prefills)
    p = plan_of(wl)
    assert p.launches() == (True, False, False)
    h = np.frombuffer(p.host, test_plan.HEADER, count=1)[0]
    pre = np.frombuffer(p.host, test_plan.TILE, count=int(h["n_prefill_tiles"]), offset=int(h["off_prefill_tiles"]))
    chunk, got = blocks(len(pre), int(h["prefill_rows"]), 256)
    assert (chunk > 0) == ordered
    head = (pre["item"].astype(np.int64) * 32 + pre["q_head0"])[got // 2]
    rounds = head[:len(head) // 256 * 256].reshape(-1, 32, 8)  # block b runs on XCD b mod 8
    assert np.mean([len(np.unique(r[:, x])) for r in rounds for x in range(8)]) <= heads


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [128, 64])
def test_ordered_launch_matches(dev, fmt, d):  # noqa: F811
    """A plan for few CUs, whose prefill tiles are ordered, in one launch with its decodes."""
    wl = workloads.make_workload("xcd", 2, hq=8, hkv=8, d=d, decodes=[(64, 1000)] * 20, prefills=[1100, 1030])
    p, *_ = run_case(wl, dev, fmt, num_cus=8)
    assert p.launches() == (True, False, False) and p.info.num_prefill_tiles >= 64 * (2 if d == 64 else 1)
