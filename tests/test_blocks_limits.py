"""How many query tokens the attention over selected blocks takes (no GPU): what the
header says, on both sides of it."""
from __future__ import annotations

import os
import re

import pytest

import paper_2607_26475_amd as ckv
from test_blocks_abi import FAKE, STATUS, _cache, attend, select

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    with open(os.path.join(ROOT, "include", "ckv.h")) as f:
        return re.sub(r"\s*\n \* ?", " ", f.read())


@pytest.mark.parametrize("heads", [1, 3, 8])
def test_tokens_times_heads(heads):
    text = _header()
    at = text.index("attention over selected blocks ---")
    assert "num_tokens * Hkv < 2^24 (CKV_EUNSUPPORTED otherwise" in text[at:at + 1500]
    most = ((1 << 24) - 1) // heads
    s = ckv.shape_for(2, heads, heads, 64)
    assert ckv.blocks_workspace_bytes(s, 32, 4, most) >= 4 * most * heads * 2
    with pytest.raises(ckv.CkvError, match="grid too large"):
        ckv.blocks_workspace_bytes(s, 32, 4, most + 1)
    c = _cache(page_stride=heads * 16 * 128)
    for call in (select, attend):
        # (a workspace that is too small: nothing is launched)
        assert call(s=s, c=c, n=most, ws=FAKE, size=0) == STATUS["EWORKSPACE"]
        assert call(s=s, c=c, n=most + 1, ws=FAKE, size=0) == STATUS["EUNSUPPORTED"]


def test_scoring_workgroups():
    assert "pieces of 64 query rows by 1024 blocks of max_ctx" in _header()
    c = _cache(page_size=65536, head_stride=65536 * 128, page_stride=65536 * 128,
               table_stride=1 << 14)
    s = ckv.shape_for(1, 16, 1, 1 << 30)     # 2^25 blocks of 32, four tokens a piece
    most = 4 * (((1 << 24) - 1) // (1 << 15))
    assert select(s=s, c=c, n=most, ws=FAKE, size=0) == STATUS["EWORKSPACE"]
    assert select(s=s, c=c, n=most + 1, ws=FAKE, size=0) == STATUS["EUNSUPPORTED"]
