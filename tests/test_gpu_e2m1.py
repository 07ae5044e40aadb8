"""The paged cache in four bits on the device, against plain 64-bit forms
(MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from e2m1_helpers import GROUP, Pool4, e2m1_64, values4
from paged_helpers import D, HALF, SCALE, U24, rope64, rope_slack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _log(*a):
    print(*a, flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- writing and reading back ------------------------------------------------------
@pytest.mark.parametrize("page,order", [(1, "heads"), (8, "rows"), (16, "pairs"), (64, "heads"),
                                        (256, "rows")])
def test_write_stores_rows_and_leaves_the_rest(page, order):
    _log("write", page, order)
    pool = Pool4([130, 1, 40, 17], 3, page, seed=page, order=order, holes=[(2, 0)], max_ctx=300)
    g = torch.Generator().manual_seed(5)
    tokens = [(0, 0), (0, 129), (1, 0), (3, 16), (0, 64), (2, 39), (2, 0),   # the last: no page
              (0, -1), (1, 300), (4, 0), (-1, 0), (3, 290)]                    # refused or no page
    x = torch.randn((len(tokens), 6, D), generator=g)
    x = (x * torch.exp2(torch.randint(-20, 20, (len(tokens), 6, 1), generator=g).float())).to(
        torch.bfloat16)
    names = ("k", "v", "k_exps", "v_exps")
    before = {n: getattr(pool, n).cpu().clone() for n in names}
    xd = x.to(DEV)
    ckv.paged_write(pool.shape(2), pool.cache, _i32([t[0] for t in tokens]),
                    _i32([t[1] for t in tokens]), xd[:, :3], xd[:, 3:])
    after = {n: getattr(pool, n).cpu() for n in names}
    table, stored = pool.table.cpu(), 0
    want = {n: t.clone() for n, t in before.items()}
    for i, (b, p) in enumerate(tokens):
        if not (0 <= b < 4 and 0 <= p < 300) or table[b, p // page] < 0:
            continue
        stored += 1
        at = (int(table[b, p // page]), slice(None), p % page)
        want["k"][at], want["k_exps"][at] = e2m1_64(x[i, :3].double())
        want["v"][at], want["v_exps"][at] = e2m1_64(x[i, 3:].double())
    assert stored >= 4
    for n in names:
        assert torch.equal(after[n], want[n]), n


def test_rounding_and_special_rows():
    """Ties, both sides of the border where the exponent steps, zeros, bf16's
    smallest and largest, infinities and NaN, each group by itself."""
    rows = torch.zeros((12, 1, D), dtype=torch.float64)
    rows[0, 0] = (torch.arange(D) - 64) / 8.0                    # every tie, scales by group
    rows[1, 0, :8] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows[1, 0, 32:40] = -rows[1, 0, :8]
    rows[2, 0, ::32] = torch.tensor([6.0, 6.03125, 5.96875, 12.0])
    rows[2, 0, 1::32] = 1.0
    rows[3, 0, :4] = torch.tensor([math.inf, 1.0, -2.0, 0.0])    # only the first group is NaN
    rows[3, 0, 40:42] = torch.tensor([3.0, 1.0])
    rows[4, 0] = math.nan
    rows[5, 0] = -0.0
    rows[6, 0, ::32] = torch.tensor([3.3895313892515355e38, 2.0 ** 127, 1.5 * 2.0 ** 127,
                                     2.0 ** 126])
    rows[6, 0, 1::32] = 2.0 ** 125
    rows[7, 0] = (torch.arange(D) - 64.0) * 2.0 ** -133          # bf16 subnormals
    rows[8, 0, ::32] = torch.tensor([2.0 ** -126, 3 * 2.0 ** -126, 2.0 ** -123, 6 * 2.0 ** -125])
    rows[9, 0] = 1.75 * 2.0 ** torch.arange(-64, 64).double()
    rows[10, 0] = torch.linspace(-6, 6, D, dtype=torch.float64)
    rows[11, 0, 5], rows[11, 0, 77] = -math.inf, math.nan
    x = rows.to(torch.bfloat16)
    pool = Pool4([16], 1, 16, spare=0)
    xd = x.to(DEV)
    pos = torch.arange(12, dtype=torch.int32, device=DEV)
    ckv.paged_write(pool.shape(1), pool.cache, torch.zeros_like(pos), pos, xd, xd)
    codes, e = e2m1_64(x.double())
    page = int(pool.table[0, 0])
    got, ge = pool.k.cpu()[page, 0, :12], pool.k_exps.cpu()[page, 0, :12]
    assert torch.equal(ge, e[:, 0])
    fine = (e[:, 0] != 255).repeat_interleave(GROUP // 2, -1)
    assert torch.equal(got[fine], codes[:, 0][fine])
    assert torch.equal(pool.v[page, 0, :12].cpu(), got) and torch.equal(
        pool.v_exps[page, 0, :12].cpu(), ge)
    # read back: the values exactly
    kd = torch.empty((1, 1, 12, D), dtype=torch.bfloat16, device=DEV)
    vd = torch.empty_like(kd)
    ckv.paged_read(pool.shape(1), pool.cache, pool.ctx, None, None, 12, kd, vd)
    want = values4(codes[:, 0], e[:, 0])
    got = kd[0, 0].cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok]) and torch.equal(torch.signbit(got[ok]),
                                                          torch.signbit(want[ok]))


def test_every_byte_and_exponent_reads_back():
    """All 256 bytes under every exponent byte of the format (0 .. 252, 255)."""
    exps = torch.cat([torch.arange(253), torch.tensor([255])]).to(torch.uint8)
    pool = Pool4([4 * 254], 1, 16, spare=0)
    k = torch.empty_like(pool.k)
    # row (e, i): bytes 64 i .. 64 i + 63, each group with exponent e
    flat = torch.arange(256, dtype=torch.uint8).view(4, 64).repeat(254, 1)
    ex = exps.repeat_interleave(4)[:, None].expand(-1, 4)
    n = 4 * 254
    table = pool.table.cpu()[0].long()
    at = torch.arange(n)
    kc, ec = pool.k.cpu(), pool.k_exps.cpu()
    kc[table[at // 16], 0, at % 16], ec[table[at // 16], 0, at % 16] = flat, ex
    k.copy_(kc)
    e = ec.to(DEV)
    c = ckv.paged_cache_for(k, k, pool.table, e, e)
    out = torch.empty((2, 1, 1, n, D), dtype=torch.bfloat16, device=DEV)
    ckv.paged_read(pool.shape(1), c, pool.ctx, None, None, n, out[0], out[1])
    want = values4(flat, ex)
    for got in out.cpu().double():
        assert torch.equal(torch.isnan(got[0, 0]), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert torch.equal(got[0, 0][ok], want[ok])


@pytest.mark.parametrize("interleaved,rot", [(False, 128), (False, 64), (False, 36), (True, 128),
                                             (True, 20)])
def test_write_rotates(interleaved, rot):
    _log("write rope", interleaved, rot)
    pool = Pool4([70, 33], 2, 16, seed=rot)
    freq, _ = ckv.rope_frequencies(rot, 10000.0)
    rope = ckv.rope_for(freq.to(DEV), rot_dim=rot, layout=int(interleaved), scale=1.5)
    tokens = [(0, p) for p in range(70)] + [(1, p) for p in range(33)] + [(0, -1)]
    n = len(tokens)
    x = torch.randn((n, 8, D), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    xd = x.to(DEV)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    q_out = torch.empty((n, 4, D), dtype=torch.bfloat16, device=DEV)
    ckv.paged_write(pool.shape(2), pool.cache, _i32([t[0] for t in tokens]),
                    _i32([t[1] for t in tokens]), xd[:, 4:6], xd[:, 6:], rope=rope,
                    q=ckv.rows_for(xd[:, :4], q_out))
    pos = torch.tensor([t[1] for t in tokens])
    wq = rope64(q, pos, freq, rot, interleaved, False, 1.5)
    tol = rope_slack(q, rot, interleaved, 1.5) + HALF[torch.bfloat16] * wq.abs()
    assert torch.all((q_out.cpu().double() - wq).abs() <= tol)
    wk = rope64(k, pos, freq, rot, interleaved, False, 1.5)
    slack = rope_slack(k, rot, interleaved, 1.5)
    table = pool.table.cpu()
    kc, ke, vc, ve = pool.k.cpu(), pool.k_exps.cpu(), pool.v.cpu(), pool.v_exps.cpu()
    for i, (b, p) in enumerate(tokens[:-1]):
        at = (int(table[b, p // 16]), slice(None), p % 16)
        two = torch.exp2(ke[at].double() - 127)
        most = wk[i].unflatten(-1, (4, GROUP)).abs().amax(-1)
        s = slack[i].unflatten(-1, (4, GROUP)).amax(-1)
        assert torch.all(most <= 6 * two + s) and torch.all(most > 3 * two - s)
        got = values4(kc[at], ke[at]).unflatten(-1, (4, GROUP))
        w = wk[i].unflatten(-1, (4, GROUP))
        # half a step: a quarter of the unit below 1, a quarter of the leading
        # power (of a value that the fp32 slack may have moved up) beyond
        z = (w.abs() + s[..., None]) / two[..., None]
        half = torch.exp2(torch.floor(torch.log2(z.clamp(min=1.0)))) / 4 * two[..., None]
        assert torch.all((got - w).abs() <= half + s[..., None]), (b, p)
        assert torch.equal(values4(vc[at], ve[at]), values4(*e2m1_64(v[i].double())))


@pytest.mark.parametrize("interleaved,rot,scale", [(False, 128, 1.0), (True, 128, 0.75),
                                                   (False, 64, 1.0), (True, 20, 2.0 ** -120)])
def test_rotated_codes_are_those_of_64_bits(interleaved, rot, scale):
    """Codes and exponents of keys turned by near and far positions are the ones that
    the rotation in 64 bits has: its rounding, 2^-52 of an angle, meets the middle
    between two codes in about one of 10^9 elements."""
    _log("codes", interleaved, rot, scale)
    n, page, far = 600, 16, 200000
    g = torch.Generator().manual_seed(rot)
    pos = torch.randperm(far, generator=g)[:n].sort().values
    pos[0] = 0
    pages = torch.unique(pos // page)
    table = torch.full((1, far // page), -1, dtype=torch.int32)
    table[0, pages] = torch.arange(len(pages), dtype=torch.int32)
    kc, vc = (torch.zeros((len(pages), 1, page, D // 2), dtype=torch.uint8, device=DEV)
              for _ in "kv")
    ke, ve = (torch.zeros((len(pages), 1, page, 4), dtype=torch.uint8, device=DEV) for _ in "kv")
    td = table.to(DEV)
    cache = ckv.paged_cache_for(kc, vc, td, ke, ve)
    freq, _ = ckv.rope_frequencies(rot, 10000.0)
    fd = freq.to(DEV)
    rope = ckv.rope_for(fd, rot_dim=rot, layout=int(interleaved), scale=scale)
    x = torch.randn((n, 1, D), generator=g).to(torch.bfloat16)
    x[5], x[6, 0, 3], x[7, 0, 40] = 0, 2.0 ** -130, 3e38
    xd = x.to(DEV)
    ckv.paged_write(ckv.shape_for(1, 1, 1, far), cache, torch.zeros(n, dtype=torch.int32, device=DEV),
                    pos.int().to(DEV), xd, xd, rope=rope)
    codes, exps = e2m1_64(rope64(x, pos, freq, rot, interleaved, False, scale))
    at = (table[0, pos // page].long(), 0, pos % page)
    assert torch.equal(ke.cpu()[at], exps[:, 0])
    got, want = kc.cpu()[at], codes[:, 0]
    # (a zero may have either sign: one of exact terms that cancel)
    zero = values4(want, exps[:, 0]) == 0
    assert torch.equal(values4(got, exps[:, 0]), values4(want, exps[:, 0]))
    assert torch.equal(zero, values4(got, exps[:, 0]) == 0)
    assert torch.equal(values4(vc.cpu()[at], ve.cpu()[at]), values4(*e2m1_64(x[:, 0].double())))


@pytest.mark.parametrize("page,order", [(1, "rows"), (4, "heads"), (16, "pairs"), (128, "heads")])
def test_read(page, order):
    _log("read", page, order)
    pool = Pool4([200, 0, 3, 131], 2, page, seed=page + 1, order=order, holes=[(0, 1), (3, 0)],
                 max_ctx=210)
    k = 150
    g = torch.Generator().manual_seed(2)
    idx = torch.full((4, 2, k), -1, dtype=torch.int32)
    n_sel = torch.zeros((4, 2), dtype=torch.int32)
    for b, n in enumerate(pool.lens):
        for h in range(2):
            m = min(n, 100 + 20 * h)
            idx[b, h, :m] = torch.randperm(n, generator=g)[:m].sort().values.int()
            n_sel[b, h] = m
    idx[0, 0, 3] = idx[0, 0, 2]                # the same position twice
    idx[0, 1, 1], idx[0, 1, 2] = 205, 5000000  # past the length, past everything
    n_sel[3, 1] = k + 9                        # clamped (its entries are -1)
    for use_idx in (True, False):
        kd = torch.full((4, 2, k, D), 5.0, dtype=torch.bfloat16, device=DEV)
        vd = torch.full((4, 2, k, D), 6.0, dtype=torch.bfloat16, device=DEV)
        ckv.paged_read(pool.shape(1), pool.cache, pool.ctx, idx.to(DEV) if use_idx else None,
                       n_sel.to(DEV) if use_idx else None, k, kd, vd)
        for b, n in enumerate(pool.lens):
            for h in range(2):
                p = idx[b, h].long() if use_idx else torch.arange(k)
                ok = (p >= 0) & (p < n) & (torch.arange(k) < (n_sel[b, h] if use_idx else k))
                ok &= pool.there[b, p.clamp(0, pool.max_ctx - 1)]
                for got, src, fill in ((kd, pool.K, 5.0), (vd, pool.V, 6.0)):
                    got = got[b, h].cpu()
                    assert torch.all(got[~ok] == fill)
                    assert torch.equal(got[ok].double(), src[b, h, p[ok]])


# ---- scores ----------------------------------------------------------------------------
def _check_scores(pool, G, max_ctx):
    q = torch.randn((pool.B, pool.Hkv * G, D), generator=torch.Generator().manual_seed(1)).to(
        torch.bfloat16)
    scores = torch.full((pool.B, pool.Hkv, max_ctx), 9.0, device=DEV)
    ckv.paged_score_keys(pool.shape(G), pool.cache, q.to(DEV), pool.ctx, SCALE, scores)
    x = q.double().view(pool.B, pool.Hkv, G, D)
    got = scores.cpu().double()
    for b in range(pool.B):
        k, there = pool.K[b], pool.there[b]
        want = torch.matmul(x[b], k.transpose(1, 2)).amax(1) * SCALE
        # 128 fp32 sums and the scaling
        tol = 130 * U24 * torch.matmul(x[b].abs(), k.abs().transpose(1, 2)).amax(1) * SCALE
        assert torch.all(got[b, :, ~there] == -math.inf), b
        assert torch.all(((got[b] - want).abs() <= tol)[:, there]), b


@pytest.mark.parametrize("page,order,G", [(1, "heads", 4), (4, "rows", 1), (16, "pairs", 2),
                                          (32, "heads", 8), (256, "rows", 16), (2, "heads", 8)])
def test_scores(page, order, G):
    _log("scores", page, order, G)
    _check_scores(Pool4([1, 700, 0, 64, 513], 2, page, seed=G, order=order,
                        holes=[(1, 1), (1, 2), (4, 0)], max_ctx=777), G, 777)


@pytest.mark.parametrize("lens,Hkv,page,G,max_ctx", [
    ([1, 20000, 0, 64, 513], 2, 16, 4, 30000), ([1, 20000, 0, 64, 513], 2, 4, 8, 30000),
    ([900, 0, 7] * 110, 1, 64, 16, 1000), ([400] * 300, 1, 2, 1, 1100)])
def test_scores_by_ranges(lens, Hkv, page, G, max_ctx):
    """More steps than workgroups: ranges over requests and heads."""
    _log("scores by ranges", len(lens), page, G)
    _check_scores(Pool4(lens, Hkv, page, seed=3, holes=[(0, 0), (1, 3)], max_ctx=max_ctx), G,
                  max_ctx)


# ---- attention ---------------------------------------------------------------------------
def _attend(pool, G, T, q, lse=True, ws=None):
    shape = pool.shape(G)
    out = torch.full((pool.B, T, pool.Hkv * G, D), 9.0, device=DEV)
    l = torch.full((pool.B, T, pool.Hkv * G), 9.0, device=DEV) if lse else None
    ws = ckv.workspace(shape, T, ckv.ENTRY_PAGED_DECODE_ATTN) if ws is None else ws
    ckv.paged_decode_attn(shape, pool.cache, T, q.to(DEV), pool.ctx, SCALE, out, l, ws)
    return out, l


def _check_attention(pool, G, T, seed=0):
    q = torch.randn((pool.B, T, pool.Hkv * G, D), generator=torch.Generator().manual_seed(seed))
    q = q.to(torch.bfloat16)
    want, wl, tol = pool.attention(q, T)
    out, lse = _attend(pool, G, T, q)
    got, gl = out.cpu().double(), lse.cpu().double()
    none = wl == -math.inf
    assert torch.all(got[none] == 0) and torch.all(gl[none] == -math.inf)
    err = (got - want).abs().amax(-1)
    assert torch.all(err <= tol), float((err / tol.clamp(min=1e-30)).max())
    # the log-sum's error is its logits' and 2^-22 of its own size
    assert torch.all(((gl - wl).abs() <= tol + 2.0 ** -22 * wl.abs() + 1e-6)[~none])
    return q, out, lse


@pytest.mark.parametrize("page,order,G,T", [(1, "heads", 4, 1), (4, "rows", 1, 3),
                                            (16, "pairs", 2, 2), (32, "heads", 8, 2),
                                            (256, "rows", 16, 1), (64, "pairs", 4, 4)])
def test_attention(page, order, G, T):
    """Direct pieces: lengths around tiles, empty requests, holes, a request with no page."""
    _log("attention", page, order, G, T)
    lens = [1, 2, 0, 15, 16, 17, 127, 128, 129, 700, 513]
    holes = [(9, 1), (9, 2), (10, 0), (3, 0)]
    pool = Pool4(lens, 2, page, seed=page, order=order, holes=holes, max_ctx=777)
    _check_attention(pool, G, T)


@pytest.mark.parametrize("lens,Hkv,page,G,T,max_ctx", [
    ([1, 9000, 0, 64, 513], 2, 16, 4, 1, 70000), ([1, 9000, 0, 64, 513], 2, 4, 8, 2, 70000),
    ([900, 0, 7] * 60, 1, 64, 16, 1, 40000), ([20000], 1, 64, 4, 4, 20000),
    ([3000, 4001], 4, 32, 1, 1, 4001)])
def test_attention_by_ranges_and_joins(lens, Hkv, page, G, T, max_ctx):
    _log("attention by ranges", len(lens), page, G, T, max_ctx)
    pool = Pool4(lens, Hkv, page, seed=7, holes=[(0, 0)] if len(lens) > 1 else [(0, 3)],
                 max_ctx=max_ctx)
    q, out, lse = _check_attention(pool, G, T)
    again, l2 = _attend(pool, G, T, q)
    assert torch.equal(again, out) and torch.equal(l2, lse)       # the same bits
    alone, _ = _attend(pool, G, T, q, lse=False)
    assert torch.equal(alone, out)


def test_nan_group_reaches_only_its_channels():
    """A NaN group of V makes its 32 channels NaN, one of K the whole row."""
    pool = Pool4([40], 1, 16, seed=2)
    q = torch.randn((1, 1, 4, D), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    page = int(pool.table[0, 1])
    pool.v_exps[page, 0, 3, 2] = 255
    out, lse = _attend(pool, 4, 1, q)
    bad = torch.zeros(D, dtype=torch.bool)
    bad[64:96] = True
    assert torch.equal(torch.isnan(out[0, 0].cpu()), bad.expand(4, D))
    assert torch.all(torch.isfinite(lse))
    pool.k_exps[page, 0, 5, 0] = 255
    out, _ = _attend(pool, 4, 1, q)
    assert torch.all(torch.isnan(out))


def test_serving_loop_write_score_select_read_attend():
    """The operators together: a step's token is written rotated, the keys are
    scored, the best rows selected and read back, and attention over them and
    over everything run; captured once and replayed over new tokens."""
    B, H, G, n, k = 3, 2, 4, 600, 256
    pool = Pool4([n] * B, H, 16, seed=4, max_ctx=n + 40, spare=40)
    table = pool.table.clone()
    free = sorted(set(range(pool.k.shape[0])) - set(table.flatten().tolist()))
    for b in range(B):  # pages for the tokens to come
        for s in range(-(-n // 16), table.shape[1]):
            table[b, s] = free.pop()
    pool.table.copy_(table)
    shape = pool.shape(G)
    ctx = _i32([n] * B)
    g = torch.Generator().manual_seed(1)
    qkv = torch.empty((B, (G + 2) * H, D), dtype=torch.bfloat16, device=DEV)
    pos = _i32([n] * B)
    freq, _ = ckv.rope_frequencies(D, 10000.0)
    rope = ckv.rope_for(freq.to(DEV))
    q = torch.empty((B, G * H, D), dtype=torch.bfloat16, device=DEV)
    scores = torch.empty((B, H, pool.max_ctx), device=DEV)
    idx = torch.empty((B, H, k), dtype=torch.int32, device=DEV)
    n_sel = torch.empty((B, H), dtype=torch.int32, device=DEV)
    kb = torch.zeros((B, H, k, D), dtype=torch.bfloat16, device=DEV)
    vb = torch.zeros_like(kb)
    some, every = (torch.empty((B, G * H, D), device=DEV) for _ in "se")
    ws1 = ckv.workspace(shape, k, ckv.ENTRY_SELECT_TOPK)
    ws2 = ckv.workspace(shape, k, ckv.ENTRY_SPARSE_DECODE_ATTN)
    ws3 = ckv.workspace(shape, 1, ckv.ENTRY_PAGED_DECODE_ATTN)

    def step():
        ckv.paged_write(shape, pool.cache, None, pos, qkv[:, G * H:(G + 1) * H],
                        qkv[:, (G + 1) * H:], rope=rope, q=ckv.rows_for(qkv[:, :G * H], q))
        ckv.paged_score_keys(shape, pool.cache, q, ctx, SCALE, scores)
        ckv.select_topk(shape, scores, ctx, k, idx, n_sel, ws1)
        ckv.paged_read(shape, pool.cache, ctx, idx, n_sel, k, kb, vb)
        ckv.sparse_decode_attn(shape, q, kb, vb, n_sel, k, SCALE, some, ws2)
        ckv.paged_decode_attn(shape, pool.cache, 1, q, ctx, SCALE, every, None, ws3)

    graph = torch.cuda.CUDAGraph()
    for t in range(4):
        qkv.copy_(torch.randn(qkv.shape, generator=g).to(torch.bfloat16))
        pos.fill_(n + t)
        ctx.fill_(n + t + 1)
        if t == 0:
            step()
            with torch.cuda.graph(graph):
                step()
        eager = None
        if t:
            graph.replay()
            torch.cuda.synchronize()
            replayed = [x.clone() for x in (some, every, idx)]
            step()
            eager = [some, every, idx]
            assert all(torch.equal(a, b) for a, b in zip(replayed, eager)), t
        # the whole attention, from what the cache stands for
        kd = torch.empty((B, H, pool.max_ctx, D), dtype=torch.bfloat16, device=DEV)
        vd = torch.empty_like(kd)
        ckv.paged_read(shape, pool.cache, ctx, None, None, pool.max_ctx, kd, vd)
        m = n + t + 1
        K, V = kd[:, :, :m].cpu().double(), vd[:, :, :m].cpu().double()
        x = q.cpu().double().view(B, H, G, D)
        l = x @ K.transpose(2, 3) * SCALE
        d = 130 * U24 * (x.abs() @ K.abs().transpose(2, 3)).amax(-1) * SCALE
        tol = ((2 * d + (m + 64) * U24) * V.abs().amax())[..., None]
        want = torch.softmax(l, -1) @ V
        assert torch.all((every.cpu().double().view(B, H, G, D) - want).abs() <= tol)
        sel = idx.cpu().long()
        ls = l.gather(-1, sel[:, :, None].expand(-1, -1, G, -1))
        vs = V.gather(2, sel[..., None].expand(-1, -1, -1, D))
        want = torch.softmax(ls, -1) @ vs
        # (the sparse attention's weights are within 2^-18 of theirs)
        assert torch.all((some.cpu().double().view(B, H, G, D) - want).abs() <=
                         tol + 2.0 ** -17 * V.abs().amax())
