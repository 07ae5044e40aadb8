"""The attention's join inside a launch, call after call on one workspace (MI355X
only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D, SCALE, Pool
from test_gpu_paged import _attend, _check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _shrunk(lens, i):
    return [max(n - 100 * (i * (j + 1) % 23), 0) for j, n in enumerate(lens)]


def test_shrunk_calls_are_their_own():
    """Calls of growing and shrinking contexts back to back, two shapes in turn on a
    workspace: every one against the 64-bit form, and the same bits as on a
    workspace that no call has used."""
    pools = [Pool([2000, 64, 700], 2, 16, "bf16", seed=1), Pool([1, 500], 4, 32, "e4m3", seed=2)]
    all_there = [p.there for p in pools]
    lens = [p.lens for p in pools]
    ws = ckv.workspace(pools[0].shape(2), 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    ws.fill_(0xFF)
    for i in range(30):
        for p, there, full in zip(pools, all_there, lens):
            p.lens = full if i % 3 == 0 else _shrunk(full, i)
            p.there = there & (torch.arange(p.max_ctx) < torch.tensor(p.lens)[:, None])
            p.ctx.copy_(torch.tensor(p.lens, dtype=torch.int32))
            q, out, lse = _attend(p, 2, 1, seed=3, ws=ws)
            _check_attention(p, q, out, lse, 1)
            _, fresh, flse = _attend(p, 2, 1, seed=3)
            assert torch.equal(out, fresh) and torch.equal(lse, flse), (i, p.lens)


def test_replays_of_shrinking_contexts():
    """A captured call, replayed while contexts shrink and grow and other calls use
    the workspace between: the bits of an eager call on a workspace of its own."""
    pool = Pool([2000, 64, 700, 1300], 2, 16, "bf16", seed=4)
    s = pool.shape(4)
    ws = ckv.workspace(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    own = ckv.workspace(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    g = torch.Generator().manual_seed(5)
    q = torch.randn((4, 1, 8, D), generator=g).to(torch.bfloat16).to(DEV)
    out, want = torch.empty((4, 1, 8, D), device=DEV), torch.empty((4, 1, 8, D), device=DEV)
    lse, wlse = torch.empty((4, 1, 8), device=DEV), torch.empty((4, 1, 8), device=DEV)

    def call(o, l, w):
        ckv.paged_decode_attn(s, pool.cache, 1, q, pool.ctx, SCALE, o, l, w)

    call(out, lse, ws)                # loads the kernel before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call(out, lse, ws)
    full = pool.lens
    for i in range(20):
        pool.ctx.copy_(torch.tensor(_shrunk(full, i) if i % 4 else full, dtype=torch.int32))
        if i % 5 == 2:
            call(want, wlse, ws)      # an eager call of another tag on the graph's workspace
        if i % 7 == 3:
            ws.fill_(i)               # its contents do not matter
        out.fill_(math.nan)
        lse.fill_(math.nan)
        graph.replay()
        call(want, wlse, own)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wlse), i
