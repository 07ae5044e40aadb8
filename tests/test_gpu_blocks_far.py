"""Four-bit pages and attention over selected blocks far out: rows past 2^32 bytes,
contexts of millions of positions of which few pages are kept (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from blocks_helpers import attend64
from e2m1_helpers import e2m1_64, values4
from paged_helpers import D, SCALE, Pool, e4m3_64, values
from test_gpu_paged_far import _check_attention, _check_scores

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _log(*a):
    print(*a, flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _stored(x, kind):
    """What a cache holds of bf16 rows, in fp64."""
    return x.double() if kind == "bf16" else values(*e4m3_64(x.double())) if kind == "e4m3" \
        else values4(*e2m1_64(x.double()))


def _far_pool(lens, H, page, kind, far):
    """A pool whose pages ("page") or heads ("head") lie past 4 GiB from each other."""
    row = {"bf16": 2 * D, "e4m3": D, "e2m1": D // 2}[kind]   # bytes
    near, gap = page * row * 2, 2 ** 32 + 8 * row             # K, then V beside it
    strides = (gap, near, row, 1) if far == "page" else (near, gap, row, 1)
    P = 3 if far == "page" else 8
    buf = torch.empty(2 * gap + near * 8, dtype=torch.uint8, device=DEV)
    p = Pool.__new__(Pool)
    p.lens, p.B, p.Hkv, p.page, p.kind, p.max_ctx = lens, len(lens), H, page, kind, max(lens)
    p.k, p.v = (buf.as_strided((P, H, page, row), strides, at) for at in (0, page * row))
    if kind == "bf16":
        p.k, p.v = (buf.view(torch.bfloat16).as_strided(
            (P, H, page, D), tuple(s // 2 for s in strides[:3]) + (1,), at)
            for at in (0, page * D))
    slots = [(b, s) for b, n in enumerate(lens) for s in range(-(-n // page))]
    assert len(slots) <= P
    table = torch.full((p.B, -(-p.max_ctx // page)), -1, dtype=torch.int32)
    for i, (b, s) in enumerate(slots):
        table[b, s] = P - 1 - i
    p.table = table.to(DEV)
    p.k_exps = p.v_exps = None
    if kind != "bf16":
        size = (P, H, page) if kind == "e4m3" else (P, H, page, 4)
        p.k_exps, p.v_exps = (torch.full(size, 255, dtype=torch.uint8, device=DEV) for _ in "kv")
    p.ctx = _i32(lens)
    p.there = torch.arange(p.max_ctx) < torch.tensor(lens)[:, None]
    p.cache = ckv.paged_cache_for(p.k, p.v, p.table, p.k_exps, p.v_exps)
    return p


def _write(pool, G, seed):
    """Rows of every position, written; the pool's K and V are what it then holds."""
    at = [(b, p) for b, n in enumerate(pool.lens) for p in range(n)]
    g = torch.Generator().manual_seed(seed)
    kv = torch.randn((2, len(at), pool.Hkv, D), generator=g).to(torch.bfloat16)
    ckv.paged_write(pool.shape(G), pool.cache, _i32([b for b, _ in at]), _i32([p for _, p in at]),
                    kv[0].to(DEV), kv[1].to(DEV))
    pool.K, pool.V = (torch.zeros((pool.B, pool.Hkv, pool.max_ctx, D), dtype=torch.float64)
                      for _ in "kv")
    for x, rows in zip(kv, (pool.K, pool.V)):
        for b, r in enumerate(_stored(x, pool.kind).split(pool.lens)):
            rows[b, :, :pool.lens[b]] = r.transpose(0, 1)


@pytest.mark.parametrize("far,page,H", [("page", 16, 2), ("page", 2, 1), ("head", 16, 3),
                                        ("head", 64, 2)])
def test_four_bit_rows_past_4_gib(far, page, H):
    """Written, scored, attended over and read back."""
    _log("far e2m1", far, page, H)
    lens, G = [2 * page, page - 1], 4
    pool = _far_pool(lens, H, page, "e2m1", far)
    _write(pool, G, page)
    K, V = ([rows[b, :, :n] for b, n in enumerate(lens)] for rows in (pool.K, pool.V))
    where = [torch.arange(n) for n in lens]
    q = torch.randn((2, 1, G * H, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    _check_scores(pool, G, where, K, q[:, 0])
    _check_attention(pool, G, 1, K, V, where, q)
    dst = torch.full((2, 2, H, max(lens), D), 5.0, dtype=torch.bfloat16, device=DEV)
    ckv.paged_read(pool.shape(G), pool.cache, pool.ctx, None, None, max(lens), dst[0], dst[1])
    for got, want in zip(dst.cpu().double(), (K, V)):
        for b, n in enumerate(lens):
            assert torch.equal(got[b, :, :n], want[b])
            assert torch.all(got[b, :, n:] == 5.0)


def _check_blocks(pool, G, block, k, req, pos, q, some, where=None):
    """Landmarks, and attention over the blocks that the selection names, against the
    plain forms; returns the landmarks and the names."""
    H, n = pool.Hkv, len(req)
    s = pool.shape(G)
    nb = -(-pool.max_ctx // block)
    marks = torch.zeros((pool.B, H, nb, D), dtype=torch.bfloat16, device=DEV)
    ckv.paged_landmarks(s, pool.cache, block, pool.ctx, marks)
    idx = torch.full((n, H, k), 99, dtype=torch.int32, device=DEV)
    out = torch.full((n, G * H, D), 9.0, device=DEV)
    lse = torch.full((n, G * H), 9.0, device=DEV)
    ws = ckv.blocks_workspace(s, block, k, n)
    r, p, qd = _i32(req), _i32(pos), q.to(DEV)
    ckv.select_blocks(s, pool.cache, block, k, r, p, qd, marks, idx, ws)
    ckv.profile_begin()
    ckv.paged_block_attn(s, pool.cache, block, k, r, p, qd, idx, SCALE, out, lse, ws)
    ran = ckv.profile_end()
    idx = idx.cpu()
    want, wl, tol = attend64(pool, block, [req[i] for i in some], [pos[i] for i in some], q[some],
                             idx[some])
    err = (out.cpu().double()[some] - want).abs().amax(-1)
    assert torch.all(err <= tol), float((err / tol).max())
    gl = lse.cpu().double()[some]
    assert torch.all((gl - wl).abs() <= tol + 2.0 ** -22 * wl.abs() + 1e-6)
    return marks.cpu(), idx, ran


@pytest.mark.parametrize("kind,far,page,H,G,repeat", [
    ("bf16", "page", 64, 2, 4, 1), ("e4m3", "page", 64, 2, 2, 1), ("e2m1", "head", 64, 2, 4, 1),
    ("bf16", "head", 64, 3, 1, 1), ("bf16", "page", 64, 2, 16, 12), ("bf16", "head", 64, 2, 16, 12)])
def test_blocks_past_4_gib(kind, far, page, H, G, repeat):
    """Landmarks and attention over rows past 2^32 bytes, of few tokens and of many."""
    _log("far blocks", kind, far, page, H, G, repeat)
    lens = [2 * page, page - 1]
    pool = _far_pool(lens, H, page, kind, far)
    _write(pool, G, H)
    at = [(b, p) for b, n in enumerate(lens) for p in range(n)] * repeat
    q = torch.randn((len(at), G * H, D), generator=torch.Generator().manual_seed(3))
    q = q.to(torch.bfloat16)
    some = list(range(0, len(at), max(1, len(at) // 90)))
    marks, idx, ran = _check_blocks(pool, G, 32, 5, [b for b, _ in at], [p for _, p in at], q, some)
    many = repeat > 1
    assert ("block_many" in ran) == many and ("block_attn" in ran) != many
    for b, n in enumerate(lens):
        for j in range(-(-n // 32)):
            want = pool.K[b, :, 32 * j:min(32 * (j + 1), n)].mean(1).to(torch.bfloat16)
            assert torch.equal(marks[b, :, j], want), (b, j)
    for t in some:
        j = at[t][1] // 32
        assert idx[t].tolist() == [[*range(j + 1), *[-1] * (4 - j)]] * H


class _Sparse(Pool):
    """A pool of few kept pages of contexts of millions of positions; K and V hold the
    kept blocks' positions only."""

    def __init__(self, lens, kept, page, kind, seed):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.B, self.Hkv, self.page, self.kind = lens, len(lens), 1, page, kind
        self.max_ctx = max(lens)
        P = sum(map(len, kept)) + 1
        self.pages = torch.full((self.B, -(-self.max_ctx // page)), -1, dtype=torch.int32)
        order = torch.randperm(P - 1, generator=g) + 1   # page 0 is nobody's
        for i, (b, s) in enumerate((b, s) for b in range(self.B) for s in kept[b]):
            self.pages[b, s] = int(order[i])
        x = torch.randn((2, P, 1, page, D), generator=g).to(torch.bfloat16)
        self.rows = _stored(x, kind)
        exps = (None, None)
        if kind == "bf16":
            x[:, 0] = math.nan
            codes = x.to(DEV)
        else:
            codes, e = (e4m3_64 if kind == "e4m3" else e2m1_64)(x.double())
            e[:, 0] = 255
            codes, exps = codes.to(DEV), e.to(DEV)
        self.k, self.v, self.k_exps, self.v_exps = codes[0], codes[1], exps[0], exps[1]
        self.table, self.ctx = self.pages.to(DEV), _i32(lens)
        self.cache = ckv.paged_cache_for(self.k, self.v, self.table, self.k_exps, self.v_exps)

    def at(self, b, p):
        """K and V of positions p of request b, which are there."""
        i = (self.pages[b, p // self.page].long(), 0, p % self.page)
        return self.rows[0][i], self.rows[1][i]


@pytest.mark.parametrize("kind,page,block", [("bf16", 64, 64), ("e4m3", 16, 256), ("e2m1", 64, 32),
                                             ("e2m1", 16, 128)])
def test_blocks_of_long_contexts_that_keep_few_pages(kind, page, block):
    """Millions of positions, most of them evicted: landmarks of what is there, the
    selection over tens of thousands of blocks, attention over what it names."""
    _log("kept", kind, page, block)
    lens = [2300001, 1500007]
    last = [-(-n // page) - 1 for n in lens]
    kept = [sorted({0, 5, 20000 * 8 // page, last[0] // 2, *range(last[0] - 9, last[0] + 1)}),
            [last[1]]]
    pool = _Sparse(lens, kept, page, kind, page + block)
    G, k = 4, 4
    s, nb = pool.shape(G), -(-pool.max_ctx // block)
    marks = torch.full((2, 1, nb, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ckv.paged_landmarks(s, pool.cache, block, pool.ctx, marks)
    got = marks.cpu()
    there = [torch.cat([torch.arange(x * page, min((x + 1) * page, lens[b])) for x in kept[b]])
             for b in range(2)]
    touched = torch.zeros((2, nb), dtype=torch.bool)
    for b in range(2):
        for j in torch.unique(there[b] // block).tolist():
            p = there[b][there[b] // block == j]
            touched[b, j] = True
            assert torch.equal(got[b, 0, j], pool.at(b, p)[0].mean(0).to(torch.bfloat16)), (b, j)
    assert torch.all(got[:, 0][~touched] == 7.0)
    # tokens at the ends, in the middle, at the start; one of a context of one page
    tokens = [(0, lens[0] - 1), (0, lens[0] - 2), (0, last[0] // 2 * page + 3), (0, 1),
              (1, lens[1] - 1), (0, last[0] * page - 1)]
    q = torch.randn((len(tokens), G, D), generator=torch.Generator().manual_seed(page))
    q = q.to(torch.bfloat16)
    idx = torch.full((len(tokens), 1, k), 99, dtype=torch.int32, device=DEV)
    out = torch.full((len(tokens), G, D), 9.0, device=DEV)
    lse = torch.full((len(tokens), G), 9.0, device=DEV)
    ws = ckv.blocks_workspace(s, block, k, len(tokens))
    r, p, qd = _i32([b for b, _ in tokens]), _i32([x for _, x in tokens]), q.to(DEV)
    ckv.select_blocks(s, pool.cache, block, k, r, p, qd, marks, idx, ws)
    ckv.paged_block_attn(s, pool.cache, block, k, r, p, qd, idx, SCALE, out, lse, ws)
    for t, (b, x) in enumerate(tokens):
        own = x // block
        j = torch.nonzero(touched[b, :own]).flatten()
        best = (got[b, 0, j].double() @ q[t].double().T).amax(-1)
        order = torch.sort(best, descending=True, stable=True).indices[:k - 1]
        names = sorted(j[order].tolist()) + [own]
        assert idx[t, 0].tolist() == names + [-1] * (k - len(names)), t
        pos = there[b][torch.isin(there[b] // block, torch.tensor(names)) & (there[b] <= x)]
        K, V = pool.at(b, pos)
        l = q[t].double() @ K.T * SCALE
        d = 130 * 2.0 ** -24 * (q[t].double().abs() @ K.abs().T).amax(-1) * SCALE
        tol = (2 * d + (len(pos) + 64) * 2.0 ** -24) * V.abs().max()
        assert torch.all((out[t].cpu().double() - torch.softmax(l, -1) @ V).abs().amax(-1) <= tol), t
        wl = torch.logsumexp(l, -1)
        assert torch.all((lse[t].cpu().double() - wl).abs() <= tol + 2.0 ** -22 * wl.abs() + 1e-6)
