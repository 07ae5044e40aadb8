"""Rebuilt keys past bf16's range against the oracle (MI355X only)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_26475_amd as ckv
import synth
from helpers import device, orc, u16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [3, 40])
def test_rebuilt_keys_past_the_largest_bf16(rank):
    """Products of factors around 2^128: infinite from halfway past the largest bf16
    on, with their signs, in tiles and key by key."""
    print("range", rank, flush=True)
    dev, w = device(), synth.WORKLOADS["tiny"]
    B, Hq, Hkv, d, k, n = w.batch, w.q_heads, w.kv_heads, w.head_dim, w.k, w.max_ctx
    u_fac, w_fac = synth.low_rank_factors(w, rank, seed=2, device=dev)
    power = torch.arange(n, device=dev) % 9 - 4
    u_fac = torch.ldexp(u_fac.float(), (64 + power)[:, None]).to(torch.bfloat16)
    w_fac = torch.ldexp(w_fac.float(), torch.tensor(64, device=dev)).to(torch.bfloat16)
    idx = np.broadcast_to(np.arange(k, dtype=np.int32), (B, Hkv, k)).copy()
    cnt = np.full((B, Hkv), k, np.int32)
    k_dst = torch.zeros((B, Hkv, k, d), dtype=torch.int16, device=dev)
    ckv.reconstruct_keys(ckv.shape_for(B, Hq, Hkv, n), rank, u_fac, w_fac,
                         torch.from_numpy(idx).to(dev), torch.from_numpy(cnt).to(dev), k, k_dst)
    got = k_dst.cpu().numpy().view(np.uint16)
    o = orc()
    want = o.reconstruct_keys(o.shape(B, Hq, Hkv, d, n), rank, u16(u_fac), u16(w_fac), idx, cnt, k)
    past = (want & 0x7fff) == 0x7f80
    assert past.any() and not past.all()
    assert np.array_equal(got, want)
