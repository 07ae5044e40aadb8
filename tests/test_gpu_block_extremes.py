"""Attention over selected blocks at the ends of its types' ranges (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

from blocks_helpers import landmarks64, select64
from paged_helpers import D
from test_gpu_blocks import DEV, Call, _i32, make

pytestmark = pytest.mark.gpu


def _put(pool, what, p, value, byte):
    """Position p of request 0 of every head of an e4m3 pool: `value` [D] (multiples of
    codes) with exponent byte `byte`, on the device and in the plain form."""
    code = value.float().to(torch.float8_e4m3fn)
    page = int(pool.table[0, p // pool.page])
    getattr(pool, what)[page, :, p % pool.page] = code.view(torch.uint8).to(DEV)
    getattr(pool, what + "_exps")[page, :, p % pool.page] = byte
    getattr(pool, what.upper())[0, :, p] = code.double() * 2.0 ** (byte - 127)


def test_landmarks_past_the_largest_bf16():
    """Means of e4m3 keys up to 448 * 2^127: to the nearest bf16, infinite from
    halfway past the largest one on, with their signs."""
    block = 32
    pool = make("e4m3", [16 * block], 2, 16, seed=1)
    # 2^127 times: the largest bf16 is 2 - 2^-7, the middle to 2 is 2 - 2^-8
    sums = [(2.0, 32), (2.0, 31), (2.0, 30), (2.0, 29), (1.875, 32), (2.125, 32)]
    for j, (x, m) in enumerate(sums):
        for i in range(block):
            v = torch.full((D,), x if i < m else 1.875, dtype=torch.float64)
            v[::2] = -v[::2]
            v[5] = 0.25
            _put(pool, "k", j * block + i, 128 * v, 247)
    for j, byte in enumerate(range(247, 255), len(sums)):
        for i in range(block):
            v = torch.arange(D, dtype=torch.float64) % 9 - 4
            v[7] = (-1.0) ** byte * (448 if i % 2 else 416)
            _put(pool, "k", j * block + i, v, byte)
    _put(pool, "k", 14 * block + 3, torch.full((D,), math.nan), 254)
    c = Call(pool, 4, block, 5, 1)
    c.landmarks()
    got, want = c.marks.cpu(), landmarks64(pool, block)
    assert torch.isinf(want).sum() > 100 and torch.isnan(want).any()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])
    # and what is selected by them
    q = torch.randn((1, 8, D), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    c.select(_i32([0]), _i32([16 * block - 1]), q.to(DEV))
    assert torch.equal(c.idx.cpu(), select64(pool, block, 5, [0], [16 * block - 1], q, want))
