"""Four-bit rows of bf16's subnormal numbers (MI355X only)."""
from __future__ import annotations

import pytest
import torch

import paper_2607_26475_amd as ckv
from e2m1_helpers import Pool4, e2m1_64
from paged_helpers import D

pytestmark = pytest.mark.gpu


def test_subnormal_rows():
    """All of bf16's subnormal numbers, of either sign, alone and beside normal ones:
    steps of 2^-126 from 2^-127 on, ties to the even code."""
    sub = torch.arange(128).double() * 2.0 ** -133
    rows = torch.stack([sub, -sub, sub.flip(0), torch.where(torch.arange(D) % 32 == 0, 2.0 ** -124, sub),
                        torch.where(torch.arange(D) % 32 == 5, -3 * 2.0 ** -126, sub),
                        sub * 2.0 ** (torch.arange(D) % 3).double()])
    x = rows[:, None].to(torch.bfloat16)
    assert torch.equal(x[:, 0].double(), rows)
    pool = Pool4([len(rows)], 1, 16, spare=0)
    pos = torch.arange(len(rows), dtype=torch.int32, device="cuda:0")
    xd = x.to("cuda:0")
    ckv.paged_write(pool.shape(1), pool.cache, torch.zeros_like(pos), pos, xd, xd)
    codes, e = e2m1_64(x.double())
    page = int(pool.table[0, 0])
    for got, ge in ((pool.k, pool.k_exps), (pool.v, pool.v_exps)):
        assert torch.equal(ge.cpu()[page, 0, :len(rows)], e[:, 0])
        assert torch.equal(got.cpu()[page, 0, :len(rows)], codes[:, 0])
