"""Block lists as a caller may write them: what is passed over stands anywhere in
them (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from blocks_helpers import attend64
from paged_helpers import D
from test_gpu_blocks import Call, _i32, _log, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _lists(own, Hkv, k, seed):
    """For each token and KV head some ascending blocks up to its own, packed to the
    front, and the same ones spread over the list: -1, blocks past its own and the block
    before once more between, in front of and behind them."""
    g = torch.Generator().manual_seed(seed)
    packed = torch.full((len(own), Hkv, k), -1, dtype=torch.int32)
    spread = packed.clone()
    for t, o in enumerate(own):
        for h in range(Hkv):
            m = int(torch.randint(0, min(k - 1, o + 1) + 1, (1,), generator=g))
            blocks = torch.randperm(min(o + 1, 9), generator=g)[:m].sort().values.int()
            m = len(blocks)
            packed[t, h, :m] = blocks
            at = torch.randperm(k, generator=g)[:m].sort().values
            fill = torch.randint(0, 3, (k,), generator=g)
            row = torch.where(fill == 1, o + 1 + torch.randint(0, 1 << 20, (k,), generator=g), -1)
            row[at] = blocks.long()
            last = -1
            for i in range(k):
                if i in at:
                    last = int(row[i])
                elif fill[i] == 2:
                    row[i] = last
            spread[t, h] = row.int()
    return packed, spread


@pytest.mark.parametrize("kind,new,Hkv,G", [
    ("bf16", 9, 2, 4), ("e4m3", 70, 1, 1), ("e2m1", 70, 2, 8), ("e2m1", 3, 2, 2),
    ("bf16", 800, 2, 16), ("bf16", 1030, 2, 16), ("bf16", 1030, 8, 4)])
def test_what_is_passed_over_may_stand_anywhere(kind, new, Hkv, G):
    """Tokens of a tile whose lists name the same blocks at different places: the
    output is that of the packed lists, bit by bit, which is the plain form's."""
    _log("spread lists", kind, new, Hkv, G)
    n, block, k = max(300, new + 40), 32, 12
    pool = make(kind, [n], Hkv, 16, seed=new)
    pos = torch.arange(n - new, n, dtype=torch.int32)
    packed, spread = _lists((pos // block).tolist(), Hkv, k, new + G)
    assert not torch.equal(packed, spread)
    q = torch.randn((new, G * Hkv, D), generator=torch.Generator().manual_seed(2))
    q = q.to(torch.bfloat16)
    got = []
    for idx in (packed, spread):
        c = Call(pool, G, block, k, new)
        c.idx.copy_(idx)
        c.attend(torch.zeros_like(pos).to(DEV), pos.to(DEV), q.to(DEV))
        got += [c.out.cpu(), c.lse.cpu()]
    some = sorted({*range(0, new, max(1, new // 60)), new - 1})
    out, lse, tol = attend64(pool, block, [0] * len(some), pos[some].tolist(), q[some],
                             packed[some])
    assert torch.all((got[0][some].double() - out).abs().amax(-1) <= tol)
    assert torch.equal(got[1][some] == -math.inf, lse == -math.inf)
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


@pytest.mark.parametrize("lists", [([0, 3], [-1, 3]), ([-1, 3], [0, 3]), ([3, -1], [-1, 3]),
                                   ([-1, 3], [-1, 3]), ([9, 3], [0, 3])])
def test_two_tokens_of_a_tile(lists):
    """Of two tokens next to each other one names a block behind an entry that is
    passed over."""
    pool = make("e2m1", [130], 1, 16, seed=1)
    pos = [128, 129]
    q = torch.randn((2, 4, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    idx = torch.tensor(lists, dtype=torch.int32)[:, None]
    c = Call(pool, 4, 32, 2, 2)
    c.idx.copy_(idx)
    c.attend(_i32([0, 0]), _i32(pos), q.to(DEV))
    out, lse, tol = attend64(pool, 32, [0, 0], pos, q, idx)
    assert torch.all((c.out.cpu().double() - out).abs().amax(-1) <= tol)
    assert torch.all((c.lse.cpu().double() - lse).abs() <= tol + 1e-6 + 2.0 ** -22 * lse.abs())


def test_debug_mode_names_a_list_that_does_not_ascend():
    pool = make("bf16", [300], 2, 16, seed=1)
    q = torch.zeros((3, 2, D), dtype=torch.bfloat16, device=DEV)
    c = Call(pool, 1, 32, 4, 3)
    req, pos = _i32([0, 0, 0]), _i32([299, 200, -1])
    good = [[[0, 3, 3, 9], [-1, 4, -1, 5]], [[3, 8, 2, -1], [-1, -1, -1, -1]],
            [[5, 4, 3, 2], [9, 8, 7, 6]]]   # 8 is past the second's own; the third is padding
    c.idx.copy_(_i32(good))
    ckv.set_debug(True)
    try:
        with pytest.raises(ckv.CkvError, match=r"idx\[1\]\[0\] do not ascend"):
            c.attend(req, pos, q)
        c.idx[1, 0, 0] = 1
        c.attend(req, pos, q)
        c.idx[1, 1, 0], c.idx[1, 1, 3] = 6, 5
        c.idx[2, 1, 0] = 1
        with pytest.raises(ckv.CkvError, match=r"idx\[1\]\[1\] do not ascend"):
            c.attend(req, pos, q)
    finally:
        ckv.set_debug(False)
