"""The paged cache far out: rows past 2^32 bytes, contexts of millions of
positions of which few are kept, tables inside wider ones, and calls that run
beside each other (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D, HALF, SCALE, U24, Pool, e4m3_64, rope64, rope_slack, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _far_pool(lens, H, page, kind, far):
    """A pool whose pages ("page") or heads ("head") lie 4 GiB apart, empty."""
    size = 2 if kind == "bf16" else 1
    near = page * D * 2                      # K, then V beside it, in elements
    gap = 2 ** 32 // size + 8 * D            # past 4 GiB, a multiple of 16 bytes
    strides = (gap, near, D, 1) if far == "page" else (near, gap, D, 1)
    P = 3 if far == "page" else 8
    last = 2 * gap + near * 8
    buf = torch.empty(last * size, dtype=torch.uint8, device=DEV)
    if kind == "bf16":
        buf = buf.view(torch.bfloat16)
    p = Pool.__new__(Pool)
    p.lens, p.B, p.Hkv, p.page, p.kind = lens, len(lens), H, page, kind
    p.max_ctx = max(lens)
    p.k = buf.as_strided((P, H, page, D), strides)
    p.v = buf.as_strided((P, H, page, D), strides, page * D)
    per = -(-p.max_ctx // page)
    slots = [(b, s) for b, n in enumerate(lens) for s in range(-(-n // page))]
    assert len(slots) <= P
    # inside a wider table, whose other entries lead nowhere
    wide = torch.full((p.B, per + 7), 2 ** 30, dtype=torch.int32)
    for i, (b, s) in enumerate(slots):
        wide[b, 4 + s] = P - 1 - i
    p.table = wide.to(DEV)[:, 4:4 + per]
    p.k_exps = p.v_exps = None
    if kind == "e4m3":
        p.k_exps, p.v_exps = (torch.full((P, H, page), 255, dtype=torch.uint8, device=DEV)
                              for _ in range(2))
    p.ctx = torch.tensor(lens, dtype=torch.int32, device=DEV)
    p.there = torch.arange(p.max_ctx) < torch.tensor(lens)[:, None]
    p.cache = ckv.paged_cache_for(p.k, p.v, p.table, p.k_exps, p.v_exps)
    return p


def _stored(x, kind):
    """What a cache holds of bf16 rows, in fp64."""
    return x.double() if kind == "bf16" else values(*e4m3_64(x.double()))


def _check_scores(pool, G, pos, K, q):
    """Scores of positions pos [m] of each request (K [B][H][m][D], fp64)."""
    B, H = pool.B, pool.Hkv
    scores = torch.full((B, H, pool.max_ctx), 9.0, device=DEV)
    ckv.paged_score_keys(pool.shape(G), pool.cache, q.to(DEV), pool.ctx, SCALE, scores)
    got = scores.cpu()
    for b in range(B):
        m = pos[b].numel()
        x, k = q[b].double().view(H, G, D), K[b]
        want = torch.matmul(x, k.transpose(1, 2)).amax(1) * SCALE
        tol = 130 * U24 * SCALE * torch.matmul(x.abs(), k.abs().transpose(1, 2)).amax(1)
        assert torch.all((got[b][:, pos[b]].double() - want).abs() <= tol), b
        assert int((got[b] != -math.inf).sum()) == H * m, b


def _check_attention(pool, G, T, K, V, pos, q):
    B, H = pool.B, pool.Hkv
    out = torch.full(q.shape, float("nan"), device=DEV)
    lse = torch.full(q.shape[:3], float("nan"), device=DEV)
    s = pool.shape(G)
    ws = ckv.workspace(s, T, ckv.ENTRY_PAGED_DECODE_ATTN)
    ckv.paged_decode_attn(s, pool.cache, T, q.to(DEV), pool.ctx, SCALE, out, lse, ws)
    out, lse = out.cpu().double(), lse.cpu().double()
    for b in range(B):
        for t in range(T):
            ok = pos[b] < pool.lens[b] - (T - 1 - t)
            for h in range(H):
                k, v, r = K[b][h, ok], V[b][h, ok], slice(h * G, (h + 1) * G)
                x = q[b, t, r].double()
                l = x @ k.T * SCALE
                # as the pools' own attention: logits' errors, then sums of m terms
                d = 130 * U24 * (x.abs() @ k.abs().T).amax(-1) * SCALE
                tol = (2 * d + (int(ok.sum()) + 64) * U24) * v.abs().max()
                want = torch.softmax(l, -1) @ v
                assert torch.all((out[b, t, r] - want).abs() <= tol[:, None]), (b, t, h)
                wl = torch.logsumexp(l, -1)
                assert torch.all((lse[b, t, r] - wl).abs() <= tol + 4 * U24 * wl.abs() + 4 * U24)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("far,page,H", [("page", 16, 2), ("page", 2, 1), ("head", 16, 3),
                                        ("head", 64, 2)])
def test_rows_past_4_gib(kind, far, page, H):
    """Written, scored, attended and read back; rows 8 GiB apart."""
    print("far", kind, far, page, H, flush=True)
    lens = [2 * page, page - 1]
    pool = _far_pool(lens, H, page, kind, far)
    g = torch.Generator().manual_seed(page)
    G, T = 4, 1
    at = [(b, p) for b, n in enumerate(lens) for p in range(n)]
    kv = torch.randn((2, len(at), H, D), generator=g).to(torch.bfloat16)
    req = torch.tensor([b for b, _ in at], dtype=torch.int32, device=DEV)
    pos = torch.tensor([p for _, p in at], dtype=torch.int32, device=DEV)
    ckv.paged_write(pool.shape(G), pool.cache, req, pos, kv[0].to(DEV), kv[1].to(DEV))
    K, V = ([r.transpose(0, 1) for r in _stored(x, kind).split(lens)] for x in kv)
    where = [torch.arange(n) for n in lens]
    q = torch.randn((2, T, G * H, D), generator=g).to(torch.bfloat16)
    _check_scores(pool, G, where, K, q[:, 0])
    _check_attention(pool, G, T, K, V, where, q)
    dst = torch.full((2, 2, H, max(lens), D), 5.0, dtype=torch.bfloat16, device=DEV)
    ckv.paged_read(pool.shape(G), pool.cache, pool.ctx, None, None, max(lens), dst[0], dst[1])
    for got, want in zip(dst.cpu().double(), (K, V)):
        for b, n in enumerate(lens):
            assert torch.equal(got[b, :, :n], want[b])
            assert torch.all(got[b, :, n:] == 5.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotated_rows_past_4_gib(dtype):
    gap = 2 ** 32 // dtype.itemsize + D
    x = torch.randn((3, 2, D), generator=torch.Generator().manual_seed(1)).to(dtype)
    buf = torch.empty(2 * gap + 2 * D, dtype=dtype, device=DEV)
    rows = buf.as_strided((3, 2, D), (gap, D, 1))
    rows.copy_(x)
    pos = torch.tensor([5, 70000, 123], dtype=torch.int32)
    freq, _ = ckv.rope_frequencies(D, 10000.0)
    r = ckv.rope_for(freq.to(DEV), dtype=ckv.ROPE_BF16 if dtype == torch.bfloat16 else ckv.ROPE_F32)
    ckv.rope_rows(r, pos.to(DEV), ckv.rows_for(rows))
    want = rope64(x, pos, freq, D, False)
    tol = rope_slack(x, D, False) + HALF[dtype] * want.abs()
    assert torch.all((rows.cpu().double() - want).abs() <= tol)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [8, 64])
def test_long_contexts_that_keep_few_pages(kind, page):
    """Millions of positions, most of them evicted: absent runs of far more than
    64 steps of a wave, a lone page among them, and one page at the end only."""
    print("kept", kind, page, flush=True)
    lens = [2300001, 1500007]
    g = torch.Generator().manual_seed(page)
    per = [-(-n // page) for n in lens]
    kept = [sorted({0, 5, 20000 * 8 // page, per[0] // 2, *range(per[0] - 6, per[0])}), [per[1] - 1]]
    P = sum(map(len, kept)) + 1
    table = torch.full((2, per[0] + 1), -1, dtype=torch.int32)
    order = torch.randperm(P - 1, generator=g) + 1    # page 0 is nobody's
    for i, (b, s) in enumerate((b, s) for b in range(2) for s in kept[b]):
        table[b, s] = int(order[i])
    x = torch.randn((2, P, 1, page, D), generator=g).to(torch.bfloat16)
    rows = _stored(x, kind)
    pool = Pool.__new__(Pool)
    pool.lens, pool.B, pool.Hkv, pool.max_ctx = lens, 2, 1, lens[0]
    if kind == "bf16":
        x[:, 0] = float("nan")
        pages, exps = x.to(DEV), (None, None)
    else:
        codes, e = e4m3_64(x.double())
        codes[:, 0], e[:, 0] = 0x7F, 255
        pages, exps = codes.to(DEV), e.to(DEV)
    pool.table, pool.ctx = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    pool.cache = ckv.paged_cache_for(pages[0], pages[1], pool.table, exps[0], exps[1])
    where, K, V = [], [], []
    for b in range(2):
        p = torch.cat([torch.arange(s * page, min((s + 1) * page, lens[b])) for s in kept[b]])
        at = (table[b, p // page].long(), 0, p % page)
        where.append(p)
        K.append(rows[0][at][None])
        V.append(rows[1][at][None])
    G, T = 8, 2
    q = torch.randn((2, T, G, D), generator=g).to(torch.bfloat16)
    _check_attention(pool, G, T, K, V, where, q)
    _check_scores(pool, G, where, K, q[:, 1])
    k = 40
    idx = torch.stack([torch.cat([w[-k // 2:], torch.arange(1000, 1000 + k)])[:k] for w in
                       (where[0], where[1].repeat(k))])[:, None].int()
    n_sel = torch.full((2, 1), k, dtype=torch.int32, device=DEV)
    kd, vd = (torch.full((2, 1, k, D), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ckv.paged_read(pool.shape(G), pool.cache, pool.ctx, idx.to(DEV), n_sel, k, kd, vd)
    for b in range(2):
        for i, p in enumerate(idx[b, 0].tolist()):
            j = torch.nonzero(where[b] == p).flatten()
            for got, src in ((kd, K), (vd, V)):
                want = src[b][0, j[0]] if j.numel() else torch.full((D,), 5.0).double()
                assert torch.equal(got[b, 0, i].cpu().double(), want), (b, p)


@pytest.mark.parametrize("lens,max_ctx", [([2001], 2001), ([9000, 700, 3, 20000], 20000)])
def test_two_streams_with_a_workspace_each(lens, max_ctx):
    """The same call running beside itself: each has its own flags, pieces and
    outputs, and gives the bits that it gives alone."""
    pool = Pool(lens, 2, 16, "bf16", seed=4, max_ctx=max_ctx)
    G, T = 4, 1
    s = pool.shape(G)
    q = torch.randn((pool.B, T, 2 * G, D), generator=torch.Generator().manual_seed(2)).to(
        torch.bfloat16).to(DEV)
    alone = torch.empty(q.shape, device=DEV)
    ckv.paged_decode_attn(s, pool.cache, T, q, pool.ctx, SCALE, alone, None,
                          ckv.workspace(s, T, ckv.ENTRY_PAGED_DECODE_ATTN))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [ckv.workspace(s, T, ckv.ENTRY_PAGED_DECODE_ATTN) for _ in range(2)]
    outs = torch.full((2, 20, *q.shape), float("nan"), device=DEV)
    torch.cuda.synchronize()
    for i in range(20):
        for j in range(2):
            ckv.paged_decode_attn(s, pool.cache, T, q, pool.ctx, SCALE, outs[j, i], None,
                                  spaces[j], stream=streams[j])
    torch.cuda.synchronize()
    assert torch.equal(outs, alone.expand_as(outs))


def test_no_tokens_and_no_requests():
    """Empty tensors, and a batch without requests whose queries are rotated all
    the same."""
    pool = Pool([40], 2, 16, "bf16", seed=1)
    was = [t.clone() for t in (pool.k, pool.v)]
    freq, _ = ckv.rope_frequencies(D, 10000.0)
    r = ckv.rope_for(freq.to(DEV))
    none = torch.empty((0, 2, D), dtype=torch.bfloat16, device=DEV)
    pos = torch.empty(0, dtype=torch.int32, device=DEV)
    ckv.rope_rows(r, pos, ckv.rows_for(none))
    ckv.paged_write(pool.shape(1), pool.cache, None, pos, none, none, r, ckv.rows_for(none))
    x = torch.randn((3, 2, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    pos = torch.tensor([7, 0, 39], dtype=torch.int32, device=DEV)
    xd, out = x.to(DEV), torch.zeros((3, 2, D), dtype=torch.bfloat16, device=DEV)
    want = torch.zeros_like(out)
    ckv.paged_write(ckv.shape_for(0, 2, 2, 40), pool.cache, torch.zeros_like(pos), pos, xd, xd, r,
                    ckv.rows_for(xd, out))
    ckv.rope_rows(r, pos, ckv.rows_for(xd, want))
    assert torch.equal(out, want) and bool((out != 0).any())
    for t, old in zip((pool.k, pool.v), was):
        assert torch.equal(t.view(torch.int16), old.view(torch.int16))
