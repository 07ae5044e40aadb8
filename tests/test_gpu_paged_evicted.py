"""Attention over caches whose pages are gone where a workgroup's piece ends
(MI355X only)."""
from __future__ import annotations

import pytest
import torch

from paged_helpers import Pool
from test_gpu_paged import _attend, _check_attention, _log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order", [(4, "heads"), (16, "heads"), (16, "rows"), (64, "pairs")])
@pytest.mark.parametrize("max_ctx", [1000, 9000])
def test_pieces_whose_tail_is_evicted(kind, page, order, max_ctx):
    """Pieces and ranges that end inside a context, whose remaining pages are all
    gone for some waves, for all of them, or but for the context's last; pools
    without a page to spare."""
    _log("evicted tails", kind, page, order, max_ctx)
    lens = [1000 - 3 * (i % 5) for i in range(40)]
    holes = []
    for b, n in enumerate(lens):
        slots = -(-n // page)
        gone = range((128 * (b % 8) + 32 * (b % 5)) // page, slots)
        holes += [(b, s) for s in gone if s < slots - 1 or b % 3]
    pool = Pool(lens, 2, page, kind, seed=page, order=order, holes=holes, spare=0,
                max_ctx=max_ctx, rows=1000)
    q, out, lse = _attend(pool, 2, 2)
    _check_attention(pool, q, out, lse, 2)
    _, again, _ = _attend(pool, 2, 2)
    assert torch.equal(out, again)


def test_one_page_of_which_nothing_is_there():
    """A pool of a single page, which no table entry leads to: every request is
    empty, whatever its length."""
    _log("one page")
    for kind in ("bf16", "e4m3"):
        lens = [400, 129, 16, 0]
        pool = Pool(lens, 1, 16, kind, holes=[(b, s) for b in range(4) for s in range(25)], spare=1)
        q, out, lse = _attend(pool, 4, 1)
        _check_attention(pool, q, out, lse, 1)
        assert torch.all(out == 0)
