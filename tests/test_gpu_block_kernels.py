"""Which attention kernel runs for the sizes that the other tests give it (MI355X
only)."""
from __future__ import annotations

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D
from test_gpu_blocks import DEV, Call, make

pytestmark = pytest.mark.gpu


def _ran(kind, n, Hkv, G, block, k, B=1):
    pool = make(kind, [n + 40] + [1] * (B - 1), Hkv, 16, seed=1)
    c = Call(pool, G, block, k, n)
    p = torch.arange(40, 40 + n, dtype=torch.int32, device=DEV)
    q = torch.randn((n, G * Hkv, D), device=DEV).to(torch.bfloat16)
    c.idx.copy_((p // block)[:, None, None].expand(-1, Hkv, k))
    ckv.profile_begin()
    c.attend(torch.zeros_like(p), p, q)
    return {name: x[0] for name, x in ckv.profile_end().items()}


@pytest.mark.parametrize("n,Hkv,G,block,k,B", [
    (1200, 2, 16, 64, 6, 3), (1050, 8, 4, 32, 17, 3), (2040, 16, 1, 128, 3, 3),
    (1050, 4, 8, 256, 2, 3), (1030, 2, 16, 64, 5, 1), (1030, 2, 16, 32, 4, 1),
    (1030, 8, 4, 32, 4, 1), (1030, 2, 16, 64, 6, 1), (1030, 8, 4, 32, 12, 1)])
def test_many_tokens_of_a_bf16_cache_are_staged(n, Hkv, G, block, k, B):
    """From 512 workgroups of 64 query rows on, the tests' sizes among them."""
    print("staged", n, Hkv, G, block, k, B, flush=True)
    assert _ran("bf16", n, Hkv, G, block, k, B) == {"block_many": 1}


@pytest.mark.parametrize("kind,n,Hkv,G", [("bf16", 800, 2, 16), ("bf16", 780, 2, 16),
                                          ("bf16", 1900, 1, 16), ("e4m3", 1030, 2, 16),
                                          ("e2m1", 1030, 2, 16)])
def test_fewer_tokens_and_codes_go_tile_by_tile(kind, n, Hkv, G):
    print("tiles", kind, n, Hkv, G, flush=True)
    assert _ran(kind, n, Hkv, G, 32, 4) == {"block_attn": 1}
