"""Debug mode's checks of the paged cache (MI355X only)."""
from __future__ import annotations

import threading

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D, SCALE, Pool

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture
def debug_mode():
    ckv.set_debug(True)
    try:
        yield
    finally:
        ckv.set_debug(False)


def test_debug_mode_over_columns_of_a_wider_table(debug_mode):
    """A table that is the last columns of a wider one: its own entries are named,
    by their own numbers; those beside it and past the lengths do not matter."""
    pool = Pool([80, 0, 65], 1, 16, "bf16")
    wide = torch.full((3, 12), 2 ** 30, dtype=torch.int32, device=DEV)
    wide[:, 4:9] = pool.table
    table = wide[:, 4:9]
    table[1:, :] = torch.where(table[1:] < 0, 2 ** 30, table[1:])   # past the lengths
    cache = ckv.paged_cache_for(pool.k, pool.v, table)
    s = pool.shape(2)
    q = torch.randn((3, 2, D), device=DEV).to(torch.bfloat16)
    a, b = torch.empty((3, 1, 80), device=DEV), torch.empty((3, 1, 80), device=DEV)
    ckv.paged_score_keys(s, cache, q, pool.ctx, SCALE, a)
    ckv.paged_score_keys(s, pool.cache, q, pool.ctx, SCALE, b)
    assert torch.equal(a, b)
    table[2, 4] = pool.k.shape[0]
    with pytest.raises(ckv.CkvError) as e:
        ckv.paged_score_keys(s, cache, q, pool.ctx, SCALE, a)
    assert e.value.status == 1 and "page_table[2][4]" in str(e.value)


def test_debug_findings_of_two_threads_stay_apart(debug_mode):
    """Threads with a stream each, one of whose tables is bad: each call's finding
    is its own."""
    pools = [Pool([90, 40], 1, 16, "bf16", seed=i) for i in range(3)]
    pools[0].table[1, 2] = 999
    pools[0].ctx[1] = 48
    pools[1].ctx[1] = 91            # of the dense entries' check
    s = pools[0].shape(2)
    q = torch.randn((2, 2, D), device=DEV).to(torch.bfloat16)
    scores = [torch.empty((2, 1, 90), device=DEV) for _ in pools]
    torch.cuda.synchronize()
    found = [[] for _ in pools]

    def run(i):
        stream = torch.cuda.Stream()
        for _ in range(150):
            try:
                ckv.paged_score_keys(s, pools[i].cache, q, pools[i].ctx, SCALE, scores[i],
                                     stream=stream)
                found[i].append("")
            except ckv.CkvError as e:
                found[i].append(str(e))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all("page_table[1][2]" in f for f in found[0])
    assert all("ctx_lens[1]" in f for f in found[1])
    assert all(f == "" for f in found[2]) and all(len(f) == 150 for f in found)
