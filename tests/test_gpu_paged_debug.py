"""Debug mode's checks of the paged cache (MI355X only)."""
from __future__ import annotations

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
