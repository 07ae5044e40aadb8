"""The paged cache and the rotary positions on the device, against plain
64-bit forms (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D, HALF, SCALE, U24, Pool, e4m3_64, rope64, rope_slack, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _log(*a):
    print(*a, flush=True)


def bits(t):
    """Equal as bytes (NaN too)."""
    return t.contiguous().view(torch.uint8).cpu()


# ---- rotary positions ------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head_dim,rot", [(128, 128), (128, 64), (128, 96), (128, 20), (128, 2),
                                          (64, 64), (8, 6), (200, 80), (1024, 1024)])
def test_rope_rows(dtype, interleaved, head_dim, rot):
    _log("rope", dtype, interleaved, head_dim, rot)
    g = torch.Generator().manual_seed(rot)
    freq, _ = ckv.rope_frequencies(rot, 500000.0)
    for n, hq, hk, inverse, scale in ((1, 1, 1, False, 1.0), (37, 5, 2, True, 1.25),
                                      (2050 if head_dim <= 128 else 3, 3, 1, False, 1.0)):
        x = torch.randn((n, hq + hk + 1, head_dim), generator=g).to(dtype)
        # angles up to 2^24: both sides' fp64 angles are within 2^-28 of them
        pos = torch.randint(-5, 2 ** 21, (n,), generator=g, dtype=torch.int32)
        pos[0] = 2 ** 24
        xd = x.to(DEV)
        q, k = xd[:, :hq], xd[:, hq:hq + hk]
        qo = torch.full((n, hq, head_dim), 7.0, dtype=dtype, device=DEV)
        ko = torch.full((n, hk, head_dim), 7.0, dtype=dtype, device=DEV)
        r = ckv.rope_for(freq.to(DEV), head_dim=head_dim, rot_dim=rot, inverse=inverse,
                         scale=scale, layout=int(interleaved),
                         dtype=ckv.ROPE_BF16 if dtype == torch.bfloat16 else ckv.ROPE_F32)
        ckv.rope_rows(r, pos.to(DEV), ckv.rows_for(q, qo), ckv.rows_for(k, ko))
        want = rope64(x, pos, freq, rot, interleaved, inverse, scale)
        got = torch.cat([qo, ko], 1).cpu().double()
        want, src = want[:, :hq + hk], x[:, :hq + hk]
        tol = rope_slack(src, rot, interleaved, scale) + HALF[dtype] * want.abs() * (
            torch.arange(head_dim) < rot)
        assert torch.all((got - want).abs() <= tol), float((got - want).abs().max())
        # in place, q alone, then k alone: the same bits, the other rows untouched
        ckv.rope_rows(r, pos.to(DEV), ckv.rows_for(q))
        assert torch.equal(bits(q), bits(qo)) and torch.equal(bits(k), bits(x[:, hq:hq + hk]))
        ckv.rope_rows(r, pos.to(DEV), ckv.rows_for(k))
        assert torch.equal(bits(k), bits(ko))
        assert torch.equal(bits(xd[:, hq + hk:]), bits(x[:, hq + hk:]))


def test_rope_inverse_is_the_gradient():
    """d/dx of sum(w * rope(x)): the inverse call on w, against the formula's
    gradient by autograd in fp64 and against differences of the call itself."""
    g = torch.Generator().manual_seed(3)
    freq, scale = ckv.rope_frequencies(48, 10000.0, ckv.ROPE_RAMP, 8.0, 4096, 1.0, 32.0)
    pos = torch.tensor([0, 3, 100000], dtype=torch.int32)
    for interleaved in (False, True):
        x = torch.randn((3, 2, 64), generator=g)
        w = torch.randn((3, 2, 64), generator=g)
        xx = x.double().requires_grad_()
        (rope64(xx, pos, freq, 48, interleaved, False, scale) * w.double()).sum().backward()
        fd = freq.to(DEV)
        back = ckv.rope_for(fd, head_dim=64, rot_dim=48, layout=int(interleaved),
                            dtype=ckv.ROPE_F32, inverse=True, scale=scale)
        there = ckv.rope_for(fd, head_dim=64, rot_dim=48, layout=int(interleaved),
                             dtype=ckv.ROPE_F32, scale=scale)
        grad = torch.empty((3, 2, 64), device=DEV)
        ckv.rope_rows(back, pos.to(DEV), ckv.rows_for(w.to(DEV), grad))
        tol = rope_slack(w, 48, interleaved, scale) + U24 * xx.grad.abs()
        assert torch.all((grad.cpu().double() - xx.grad).abs() <= tol)
        # the map is linear: a step of 1 in x moves y by its column exactly, up to
        # the rounding of the two results
        step = torch.zeros_like(x)
        step[1, 1, 5] = 1.0
        y = torch.empty((2, 3, 2, 64), device=DEV)
        for i, z in enumerate((x, x + step)):
            ckv.rope_rows(there, pos.to(DEV), ckv.rows_for(z.to(DEV), y[i]))
        y = y.cpu().double()
        diff = float(((y[1] - y[0]) * w.double()).sum())
        slack = sum(rope_slack(z, 48, interleaved, scale) + U24 * y.abs().amax(0)
                    for z in (x, x + step))[1, 1]
        # x + 1 is rounded too
        slack = float((slack * w[1, 1].double().abs()).sum()) + 2 * U24 * float(w.abs().max()) * 8
        assert abs(diff - float(xx.grad[1, 1, 5])) <= slack


def test_rope_of_one_row_for_all():
    """A source of strides 0 and a destination with heads outermost."""
    freq, _ = ckv.rope_frequencies(128, 10000.0)
    x = torch.randn((1, 1, 128), generator=torch.Generator().manual_seed(6)).to(DEV)
    y = torch.empty((3, 7, 128), device=DEV).transpose(0, 1)
    pos = torch.arange(7, dtype=torch.int32)
    ckv.rope_rows(ckv.rope_for(freq.to(DEV), dtype=ckv.ROPE_F32), pos.to(DEV),
                  ckv.rows_for(x.expand(7, 3, 128), y))
    src = x.cpu().expand(7, 3, 128)
    want = rope64(src, pos, freq, 128, False)
    assert torch.all((y.cpu().double() - want).abs() <=
                     rope_slack(src, 128, False) + U24 * want.abs())


def test_rope_undone():
    g = torch.Generator().manual_seed(4)
    freq, _ = ckv.rope_frequencies(128, 10000.0)
    x = torch.randn((50, 4, 128), generator=g)
    pos = torch.randint(0, 10 ** 6, (50,), generator=g, dtype=torch.int32).to(DEV)
    y = x.to(DEV).clone()
    for inverse, scale in ((False, 1.5), (True, 1 / 1.5)):
        ckv.rope_rows(ckv.rope_for(freq.to(DEV), dtype=ckv.ROPE_F32, inverse=inverse, scale=scale),
                      pos, ckv.rows_for(y))
    # two rotations, each within the slack of rows of the same length, and 1 / 1.5
    tol = 2 * rope_slack(x, 128, False) * 1.5 + 4 * U24 * x.abs().max()
    assert torch.all((y.cpu().double() - x.double()).abs() <= tol)


# ---- writing and reading back -------------------------------------------------------
def _written(pool, seed, tokens, G=2, rope=None, stride_pad=0):
    """Writes `tokens` (request, position) pairs of random rows; the rows."""
    g = torch.Generator().manual_seed(seed)
    n, H = len(tokens), pool.Hkv
    x = torch.randn((n, (2 + G) * H + stride_pad, D), generator=g)
    x *= torch.exp2(torch.randint(-20, 20, (n, x.shape[1], 1), generator=g).float())
    x = x.to(torch.bfloat16)
    req = torch.tensor([t[0] for t in tokens], dtype=torch.int32)
    pos = torch.tensor([t[1] for t in tokens], dtype=torch.int32)
    xd = x.to(DEV)
    q, k, v = xd[:, :G * H], xd[:, G * H:G * H + H], xd[:, G * H + H:(2 + G) * H]
    q_out = torch.full((n, G * H, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ckv.paged_write(pool.shape(G), pool.cache, req.to(DEV), pos.to(DEV), k, v, rope=rope,
                    q=ckv.rows_for(q, q_out) if rope is not None else None)
    torch.cuda.synchronize()
    return x[:, :G * H], x[:, G * H:G * H + H], x[:, G * H + H:(2 + G) * H], q_out.cpu()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order", [(1, "heads"), (8, "rows"), (16, "pairs"), (64, "heads"),
                                        (256, "rows")])
def test_write_stores_rows_and_leaves_the_rest(kind, page, order):
    _log("write", kind, page, order)
    pool = Pool([130, 1, 40, 17], 3, page, kind, seed=page, order=order, holes=[(2, 0)], max_ctx=300)
    before = [bits(t) for t in (pool.k, pool.v)]
    tokens = [(0, 0), (0, 129), (1, 0), (3, 16), (0, 64), (2, 39), (2, 0),   # the last: no page
              (0, -1), (1, 300), (4, 0), (-1, 0), (3, 290)]                    # refused or no page
    _, k, v, _ = _written(pool, 5, tokens)
    table = pool.table.cpu()
    kp, vp = pool.k.cpu(), pool.v.cpu()
    seen = torch.zeros(kp.shape[0], page, dtype=torch.bool)
    stored = 0
    for i, (b, p) in enumerate(tokens):
        if not (0 <= b < 4 and 0 <= p < 300) or table[b, p // page] < 0:
            continue
        at = (int(table[b, p // page]), slice(None), p % page)
        seen[at[0], at[2]] = True
        stored += 1
        for x, pages, exps in ((k, kp, pool.k_exps), (v, vp, pool.v_exps)):
            if kind == "bf16":
                assert torch.equal(bits(pages[at]), bits(x[i])), (b, p)
            else:
                codes, e = e4m3_64(x[i].double())
                assert torch.equal(exps.cpu()[at], e), (b, p)
                assert torch.equal(pages[at], codes), (b, p)
    assert stored >= 4
    for t, old in ((pool.k, before[0]), (pool.v, before[1])):
        new, was = bits(t).view(*t.shape[:3], -1), old.view(*t.shape[:3], -1)
        keep = ~seen[:, None].expand(t.shape[:3])
        assert torch.equal(new[keep], was[keep])


def test_e4m3_rounding_and_special_rows():
    """Ties, both sides of the border where the exponent steps, subnormal codes,
    rows of zeros, of bf16's smallest and largest, infinities and NaN."""
    rows = torch.zeros((16, 1, D), dtype=torch.float64)
    rows[1, 0, :3] = torch.tensor([448.0, -448.0, 1.0625])          # 1.0625: a tie
    rows[2, 0, :3] = torch.tensor([450.0, 1.0, 2.0 ** -9])
    rows[3, 0] = torch.arange(D) * 2.0 ** -3 - 8
    rows[4, 0] = (torch.arange(D) - 64.0) * 2.0 ** -133              # bf16 subnormals
    rows[5, 0, 5] = 2.0 ** -133
    rows[6, 0, :2] = torch.tensor([3.3895313892515355e38, -1.0])
    rows[7, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 2.0])
    rows[8, 0] = math.nan
    rows[9, 0] = -0.0
    rows[10, 0, :6] = torch.tensor([256.0, 0.5, 2.0 ** -7, 3 * 2.0 ** -10, 2.0 ** -10, 1.5 * 2.0 ** -9])
    rows[11, 0] = 1.75 * 2.0 ** torch.arange(-64, 64).double()
    rows[12, 0, :2] = torch.tensor([448 * 2.0 ** -127, 2.0 ** -130])
    rows[13, 0, 0] = 450 * 2.0 ** -127
    rows[14, 0] = torch.linspace(-448, 448, D)
    rows[15, 0] = torch.linspace(-17, 17, D)
    x = rows.to(torch.bfloat16)
    pool = Pool([16], 1, 16, "e4m3", spare=0)
    xd = x.to(DEV)
    pos = torch.arange(16, dtype=torch.int32, device=DEV)
    ckv.paged_write(pool.shape(1), pool.cache, torch.zeros_like(pos), pos, xd, xd)
    codes, e = e4m3_64(x.double())
    page = int(pool.table[0, 0])
    got, ge = pool.k.cpu()[page, 0], pool.k_exps.cpu()[page, 0]
    assert torch.equal(ge, e[:, 0])
    nan = codes[:, 0] == 0x7F
    assert torch.equal((got & 0x7F) == 0x7F, nan)                    # either sign's NaN
    assert torch.equal(got[~nan], codes[:, 0][~nan])
    assert torch.equal(bits(pool.v), bits(pool.k)) and torch.equal(pool.v_exps, pool.k_exps)
    # read back: the values, rounded to bf16 where they are its subnormals
    kd = torch.empty((1, 1, 16, D), dtype=torch.bfloat16, device=DEV)
    vd = torch.empty_like(kd)
    ckv.paged_read(pool.shape(1), pool.cache, pool.ctx, None, None, 16, kd, vd)
    want = values(codes[:, 0], e[:, 0]).float().to(torch.bfloat16)
    fine = ~torch.isnan(want)
    assert torch.equal(torch.isnan(kd[0, 0].cpu()), ~fine)
    assert torch.equal(kd[0, 0].cpu()[fine], want[fine])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("interleaved,rot", [(False, 128), (False, 64), (False, 36), (True, 128),
                                             (True, 20)])
def test_write_rotates(kind, interleaved, rot):
    _log("write rope", kind, interleaved, rot)
    pool = Pool([70, 33], 2, 16, kind, seed=rot)
    freq, _ = ckv.rope_frequencies(rot, 10000.0)
    rope = ckv.rope_for(freq.to(DEV), rot_dim=rot, layout=int(interleaved), scale=1.5)
    tokens = [(0, p) for p in range(70)] + [(1, p) for p in range(33)] + [(0, -1)]
    q, k, v, q_out = _written(pool, 9, tokens, rope=rope, stride_pad=1)
    pos = torch.tensor([t[1] for t in tokens])
    wq = rope64(q, pos, freq, rot, interleaved, False, 1.5)
    tol = rope_slack(q, rot, interleaved, 1.5) + HALF[torch.bfloat16] * wq.abs()
    assert torch.all((q_out.double() - wq).abs() <= tol)
    wk = rope64(k, pos, freq, rot, interleaved, False, 1.5)
    slack = rope_slack(k, rot, interleaved, 1.5)
    table = pool.table.cpu()
    for i, (b, p) in enumerate(tokens[:-1]):
        at = (int(table[b, p // 16]), slice(None), p % 16)
        if kind == "bf16":
            got = pool.k.cpu()[at].double()
            assert torch.equal(bits(pool.v.cpu()[at]), bits(v[i]))
            tol = slack[i] + HALF[torch.bfloat16] * wk[i].abs()
        else:
            e = pool.k_exps.cpu()[at]
            got = values(pool.k.cpu()[at], e)
            two = torch.exp2(e.double() - 127)
            most, s = wk[i].abs().amax(-1), slack[i].amax(-1)
            assert torch.all(most <= 448 * two + s) and torch.all(most > 224 * two - s)
            # half a step: 2^-4 of the value, 2^-10 of the unit below 2^-6
            tol = slack[i] + torch.maximum(2.0 ** -4 * wk[i].abs(), 2.0 ** -10 * two[:, None])
            codes, ve = e4m3_64(v[i].double())
            assert torch.equal(pool.v.cpu()[at], codes) and torch.equal(pool.v_exps.cpu()[at], ve)
        assert torch.all((got - wk[i]).abs() <= tol), (b, p)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order", [(1, "rows"), (4, "heads"), (16, "pairs"), (128, "heads")])
def test_read(kind, page, order):
    _log("read", kind, page, order)
    pool = Pool([200, 0, 3, 131], 2, page, kind, seed=page + 1, order=order,
                holes=[(0, 1), (3, 0)], max_ctx=210)
    k = 150
    g = torch.Generator().manual_seed(2)
    idx = torch.full((4, 2, k), -1, dtype=torch.int32)
    n_sel = torch.zeros((4, 2), dtype=torch.int32)
    for b, n in enumerate(pool.lens):
        for h in range(2):
            m = min(n, 100 + 20 * h)
            idx[b, h, :m] = torch.randperm(n, generator=g)[:m].sort().values.int()
            n_sel[b, h] = m
    idx[0, 0, 3] = idx[0, 0, 2]        # the same position twice
    idx[0, 1, 1], idx[0, 1, 2] = 205, 5000000  # past the length, past everything
    n_sel[3, 1] = k + 9                  # clamped (its entries are -1)
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
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order,G", [(1, "heads", 4), (4, "rows", 1), (16, "pairs", 2),
                                          (32, "heads", 8), (256, "rows", 16), (2, "heads", 8)])
def test_paged_scores(kind, page, order, G):
    _log("scores", kind, page, order, G)
    pool = Pool([1, 700, 0, 64, 513], 2, page, kind, seed=G, order=order,
                holes=[(1, 1), (1, 2), (4, 0)], max_ctx=777)
    q = torch.randn((5, 2 * G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    scores = torch.full((5, 2, 777), 9.0, device=DEV)
    ckv.paged_score_keys(pool.shape(G), pool.cache, q.to(DEV), pool.ctx, SCALE, scores)
    x = q.double().view(5, 2, G, D)
    want = torch.matmul(x, pool.K.transpose(2, 3)).amax(2) * SCALE
    tol = 130 * U24 * torch.matmul(x.abs(), pool.K.abs().transpose(2, 3)).amax(2) * SCALE
    there = pool.there[:, None].expand_as(want)
    got = scores.cpu().double()
    assert torch.all(got[~there] == -math.inf)
    assert torch.all((got - want)[there].abs() <= tol[there])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,Hkv,page,G,max_ctx", [
    ([1, 20000, 0, 64, 513], 2, 16, 4, 30000), ([1, 20000, 0, 64, 513], 2, 4, 8, 30000),
    ([900, 0, 7] * 110, 1, 64, 16, 1000), ([400] * 300, 1, 2, 1, 1100)])
def test_paged_scores_by_ranges(kind, lens, Hkv, page, G, max_ctx):
    """More steps than workgroups: ranges over requests and heads, tails filled
    in pieces."""
    _log("scores by ranges", kind, len(lens), page, G)
    B = len(lens)
    pool = Pool(lens, Hkv, page, kind, seed=3, holes=[(0, 0), (1, 3)], max_ctx=max_ctx)
    q = torch.randn((B, Hkv * G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    scores = torch.full((B, Hkv, max_ctx), 9.0, device=DEV)
    ckv.paged_score_keys(pool.shape(G), pool.cache, q.to(DEV), pool.ctx, SCALE, scores)
    got = scores.cpu().double()
    for b, n in enumerate(lens):
        x, k = q[b].double().view(Hkv, G, D), pool.K[b, :, :n]
        want = torch.matmul(x, k.transpose(1, 2)).amax(1) * SCALE if n else torch.zeros(Hkv, 0)
        tol = 130 * U24 * SCALE * torch.matmul(x.abs(), k.abs().transpose(1, 2)).amax(1) \
            if n else torch.zeros(Hkv, 0)
        there = pool.there[b, :n]
        assert torch.all((got[b, :, :n] - want)[:, there].abs() <= tol[:, there]), b
        assert torch.all(got[b, :, :n][:, ~there] == -math.inf), b
        assert torch.all(got[b, :, n:] == -math.inf), b


# ---- attention -------------------------------------------------------------------------
def _attend(pool, G, T, seed=0, lse=True, stream=None, ws=None):
    q = torch.randn((pool.B, T, G * pool.Hkv, D),
                    generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
    out = torch.full(q.shape, float("nan"), device=DEV)
    l = torch.full(q.shape[:3], float("nan"), device=DEV) if lse else None
    s = pool.shape(G)
    if ws is None:
        ws = ckv.workspace(s, T, ckv.ENTRY_PAGED_DECODE_ATTN)
        ws.fill_(0xFF)
    ckv.paged_decode_attn(s, pool.cache, T, q.to(DEV), pool.ctx, SCALE, out, l, ws, stream=stream)
    torch.cuda.synchronize()
    return q, out.cpu().double(), l.cpu().double() if lse else None


def _check_attention(pool, q, out, lse, T):
    want, wl, tol = pool.attention(q, T)
    assert torch.all((out - want).abs() <= tol[..., None]), float((out - want).abs().max())
    empty = wl == -math.inf
    assert torch.all(out[empty] == 0)
    if lse is not None:
        assert torch.equal(lse == -math.inf, empty)
        # logits within tol / max |V| of theirs, the sum within m steps, and the
        # fp32 result itself: covered by tol (max |V| >= 1) and one rounding
        assert torch.all((lse - wl)[~empty].abs() <= (tol + 4 * U24 * wl.abs() + 4 * U24)[~empty])


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order,G,T", [
    (1, "heads", 4, 1), (2, "rows", 2, 3), (8, "pairs", 8, 2), (16, "heads", 1, 1),
    (16, "rows", 16, 1), (32, "pairs", 4, 4), (64, "heads", 8, 1), (128, "rows", 1, 16),
    (1024, "heads", 2, 2)])
def test_paged_attention(kind, page, order, G, T):
    """In one launch (a workgroup for every step), and, for the same lengths in
    longer tables, by ranges with a join of their own."""
    _log("attention", kind, page, order, G, T)
    for max_ctx in (1100, 9000):
        pool = Pool(LENS, 2, page, kind, seed=G + T, order=order, max_ctx=max_ctx)
        q, out, lse = _attend(pool, G, T)
        _check_attention(pool, q, out, lse, T)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("max_ctx", [700, 9000])
def test_paged_attention_with_evicted_pages(kind, page, max_ctx):
    """Pages missing at the front, in the middle, over whole steps, everywhere,
    and the page of the newest position."""
    _log("evicted", kind, page)
    lens = [700, 300, 129, 64, 5]
    per = lambda n: -(-n // page)  # noqa: E731
    holes = [(0, s) for s in range(1, per(500))] + [(1, s) for s in range(per(300))] + \
            [(2, 0)] + [(3, per(64) - 1)]
    pool = Pool(lens, 2, page, kind, seed=page, holes=holes, max_ctx=max_ctx)
    q, out, lse = _attend(pool, 4, 2)
    _check_attention(pool, q, out, lse, 2)
    assert torch.all(out[1] == 0)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,Hkv,G,T", [
    ([40000], 1, 8, 2), ([70001, 3], 1, 1, 1), ([9000, 0, 1, 5000, 129], 2, 4, 1),
    ([5] * 300 + [0] * 20 + [700], 1, 2, 1), ([130] * 700, 1, 1, 1)])
def test_units_over_many_ranges(kind, lens, Hkv, G, T):
    """Units that many workgroups share, many units a workgroup, and both."""
    _log("ranges", kind, len(lens), max(lens))
    pool = Pool(lens, Hkv, 64 if max(lens) > 2000 else 16, kind, seed=7)
    q, out, lse = _attend(pool, G, T)
    _check_attention(pool, q, out, lse, T)


EDGES = [0, 1, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 5, 640]


@pytest.mark.parametrize("kind,page", [("bf16", 16), ("e4m3", 64), ("bf16", 4)])
@pytest.mark.parametrize("B,Hkv,G,T", [(40, 2, 2, 1), (75, 2, 1, 3), (130, 2, 4, 1), (300, 2, 1, 2),
                                       (20, 2, 16, 1)])
def test_pieces_of_several_steps(kind, page, B, Hkv, G, T):
    """A workgroup for 2, 4 and 8 steps, and for whole units, more of them than
    the device holds at once; lengths about the pieces' ends."""
    _log("pieces", kind, page, B, Hkv, G, T)
    lens = [EDGES[(5 * i + i // 14) % 14] for i in range(B)]
    holes = [(3, 0), (4, 1), (9, 0), (9, 1)]
    pool = Pool(lens, Hkv, page, kind, seed=B, holes=holes, max_ctx=1000)
    q, out, lse = _attend(pool, G, T)
    _check_attention(pool, q, out, lse, T)
    _, again, _ = _attend(pool, G, T)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind,page", [("bf16", 16), ("e4m3", 64), ("bf16", 4)])
@pytest.mark.parametrize("lens,G,T", [([4096, 1, 0, 511, 2049], 16, 1), ([8192, 3900], 4, 2),
                                      ([9000], 4, 1)])
def test_pieces_for_the_join(kind, page, lens, G, T):
    """Few units whose steps are too many to be joined one by one."""
    _log("pieces for the join", kind, page, lens, G, T)
    pool = Pool(lens, 2, page, kind, seed=G, holes=[(0, 1), (0, 2)])
    q, out, lse = _attend(pool, G, T)
    _check_attention(pool, q, out, lse, T)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,order,G,T", [
    (1, "heads", 4, 1), (2, "rows", 2, 3), (8, "pairs", 8, 2), (16, "heads", 1, 1),
    (16, "rows", 16, 1), (32, "pairs", 4, 4), (64, "heads", 8, 1), (128, "rows", 1, 16),
    (1024, "heads", 2, 2)])
def test_ranges_of_ragged_batches(kind, page, order, G, T):
    """Short contexts in long tables, more units than pieces are made for: ranges
    over requests and heads, pages missing, a join of their own."""
    _log("ragged ranges", kind, page, order, G, T)
    lens = [EDGES[i % 14] for i in range(24)] + [3000, 0, 1777, 128, 1, 2999]
    per = lambda n: -(-n // page)  # noqa: E731
    holes = [(24, s) for s in range(1, per(2000))] + [(26, s) for s in range(per(1600))] + \
            [(11, s) for s in range(per(1000))] + [(3, 0), (29, per(2999) - 1)]
    pool = Pool(lens, 2, page, kind, seed=G + T, order=order, holes=holes, max_ctx=40000, rows=3000)
    q, out, lse = _attend(pool, G, T)
    _check_attention(pool, q, out, lse, T)


def test_shared_pages_and_no_lse():
    pool = Pool([100, 90], 2, 32, "bf16", seed=3, share=True)
    q, out, _ = _attend(pool, 4, 1, lse=False)
    _check_attention(pool, q, out, None, 1)


def test_weights_keep_fp32():
    """Equal values under unequal weights: weights cut to bf16 (2^-9 of each)
    would show beside the unrounded sum that divides them."""
    n = 256
    pool = Pool([n], 1, 16, "bf16", seed=1, spare=0)
    k = torch.zeros((n, D), dtype=torch.bfloat16)
    k[:, 0] = torch.linspace(-1, 1, n).to(torch.bfloat16)
    v = torch.ones((n, D), dtype=torch.bfloat16)
    order = pool.table[0].long().cpu()
    kp, vp = pool.k.cpu(), pool.v.cpu()
    kp[order, 0], vp[order, 0] = k.view(-1, 16, D), v.view(-1, 16, D)
    pool.k.copy_(kp)
    pool.v.copy_(vp)
    q = torch.zeros((1, 1, 1, D), dtype=torch.bfloat16)
    q[..., 0] = 20.0
    out = torch.empty((1, 1, 1, D), device=DEV)
    s = pool.shape(1)
    ckv.paged_decode_attn(s, pool.cache, 1, q.to(DEV), pool.ctx, SCALE, out, None,
                          ckv.workspace(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN))
    # equal values: the weighted mean is 1 whatever the weights, up to the
    # rounding of the two sums of n fp32 terms
    assert torch.all((out.cpu().double() - 1).abs() <= 2 * n * U24)


# ---- together, streams, graphs --------------------------------------------------------
def test_decode_steps_through_all_of_them():
    """Three decode steps on a quantised cache: queries and keys rotated and
    written, then full attention, and the sparse path (scores, selection, rows
    read back, sparse attention) with a budget of everything: the same result."""
    lens, H, G, page = [45, 130, 7], 2, 4, 16
    B, Hq, max_ctx = 3, H * G, 160
    pool = Pool([max_ctx] * B, H, page, "e4m3", seed=11)   # every page allocated
    freq, _ = ckv.rope_frequencies(128, 500000.0)
    rope = ckv.rope_for(freq.to(DEV))
    s = ckv.shape_for(B, Hq, H, max_ctx)
    ws = ckv.workspace(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    ws_sel = ckv.workspace(s, max_ctx, ckv.ENTRY_SELECT_TOPK)
    ws_att = ckv.workspace(s, max_ctx, ckv.ENTRY_SPARSE_DECODE_ATTN)
    g = torch.Generator().manual_seed(12)
    for step in range(3):
        ctx = torch.tensor([n + step + 1 for n in lens], dtype=torch.int32, device=DEV)
        x = torch.randn((B, Hq + 2 * H, D), generator=g).to(torch.bfloat16).to(DEV)
        q = torch.empty((B, Hq, D), dtype=torch.bfloat16, device=DEV)
        ckv.paged_write(s, pool.cache, None, ctx - 1, x[:, Hq:Hq + H], x[:, Hq + H:], rope=rope,
                        q=ckv.rows_for(x[:, :Hq], q))
        out, lse = torch.empty((B, 1, Hq, D), device=DEV), torch.empty((B, 1, Hq), device=DEV)
        ckv.paged_decode_attn(s, pool.cache, 1, q.view(B, 1, Hq, D), ctx, SCALE, out, lse, ws)
        scores = torch.empty((B, H, max_ctx), device=DEV)
        idx = torch.empty((B, H, max_ctx), dtype=torch.int32, device=DEV)
        n_sel = torch.empty((B, H), dtype=torch.int32, device=DEV)
        kb = torch.empty((B, H, max_ctx, D), dtype=torch.bfloat16, device=DEV)
        vb, out2 = torch.empty_like(kb), torch.empty((B, Hq, D), device=DEV)
        ckv.paged_score_keys(s, pool.cache, q, ctx, SCALE, scores)
        ckv.select_topk(s, scores, ctx, max_ctx, idx, n_sel, ws_sel)
        ckv.paged_read(s, pool.cache, ctx, idx, n_sel, max_ctx, kb, vb)
        ckv.sparse_decode_attn(s, q, kb, vb, n_sel, max_ctx, SCALE, out2, ws_att)
        torch.cuda.synchronize()
        assert torch.equal(n_sel.cpu(), ctx.cpu()[:, None].expand(-1, H))
        # the host's own view of the cache as it is now
        pool.lens = ctx.tolist()
        pool.there = torch.arange(max_ctx)[None] < ctx.cpu()[:, None]
        kd, vd = torch.zeros_like(kb), torch.zeros_like(kb)  # rows past a length stay 0
        ckv.paged_read(s, pool.cache, ctx, None, None, max_ctx, kd, vd)
        pool.K, pool.V = kd.cpu().double(), vd.cpu().double()
        _check_attention(pool, q.view(B, 1, Hq, D).cpu(), out.cpu().double(), lse.cpu().double(), 1)
        want, _, tol = pool.attention(q.view(B, 1, Hq, D).cpu(), 1)
        # the sparse attention's weights carry 2^-18 of sum p |v| besides
        tol = tol[:, 0, :, None] + 2.0 ** -18 * pool.V.abs().max()
        assert torch.all((out2.cpu().double() - want[:, 0]).abs() <= tol)


def test_same_bits_again_and_on_another_stream():
    pool = Pool([3000, 70, 0, 513], 2, 16, "e4m3", seed=5)
    _, a, la = _attend(pool, 4, 2)
    _, b, lb = _attend(pool, 4, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _, c, lc = _attend(pool, 4, 2, stream=side)
    assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(la, lb) and torch.equal(la, lc)


def test_captured_step_follows_growing_contexts():
    """Two captured graphs (two layers) that share a workspace, replayed while
    lengths, tables and rows change, with eager calls between the replays."""
    H, G, page, max_ctx, B = 2, 4, 16, 400, 3
    s = ckv.shape_for(B, H * G, H, max_ctx)
    ws = ckv.workspace(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    freq = ckv.rope_frequencies(128, 10000.0)[0].to(DEV)
    rope = ckv.rope_for(freq)
    ctx = torch.tensor([1, 150, 389], dtype=torch.int32, device=DEV)
    pos = torch.empty(B, dtype=torch.int32, device=DEV)
    layers = []
    for i in range(2):
        pool = Pool([max_ctx] * B, H, page, ("bf16", "e4m3")[i], seed=20 + i)
        x = torch.empty((B, H * G + 2 * H, D), dtype=torch.bfloat16, device=DEV)
        q = torch.empty((B, H * G, D), dtype=torch.bfloat16, device=DEV)
        out = torch.empty((B, 1, H * G, D), device=DEV)
        scores = torch.empty((B, H, max_ctx), device=DEV)
        layers.append((pool, x, q, out, scores))

    def layer(i):
        pool, x, q, out, scores = layers[i]
        ckv.paged_write(s, pool.cache, None, pos, x[:, H * G:H * G + H], x[:, H * G + H:],
                        rope=rope, q=ckv.rows_for(x[:, :H * G], q))
        ckv.paged_decode_attn(s, pool.cache, 1, q.view(B, 1, H * G, D), ctx, SCALE, out, None, ws)
        ckv.paged_score_keys(s, pool.cache, q, ctx, SCALE, scores)

    for pool, x, *_ in layers:
        x.zero_()
    pos.copy_(ctx - 1)
    layer(0), layer(1)                       # loads the kernels before the capture
    torch.cuda.synchronize()
    graphs = []
    side = torch.cuda.Stream()
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer(i)
        graphs.append(graph)
    g = torch.Generator().manual_seed(30)
    for step in range(4):
        ctx.add_(2 if step else 0)
        pos.copy_(ctx - 1)
        for _, x, *_ in layers:
            x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [(bits(l[2]), bits(l[3]), bits(l[4])) for l in layers]
        for l in layers:
            l[3].fill_(7.0), l[4].fill_(7.0)
        layer(0), layer(1)
        torch.cuda.synchronize()
        for l, want in zip(layers, got):
            assert all(torch.equal(bits(t), w) for t, w in zip(l[2:], want))


def test_kernel_classes_are_timed():
    for lens, merges in (([300], 0), ([9000], 0), ([70000], 1)):  # one launch; ranges, their join
        pool = Pool(lens, 1, 16, "bf16")
        ckv.profile_begin(["paged_attn", "paged_merge"])
        _attend(pool, 1, 1)
        seen = ckv.profile_end()
        assert seen["paged_attn"][0] == 1 and seen.get("paged_merge", (0,))[0] == merges


def test_direct_join_over_and_over():
    """The hand-over flags are clear again after every call: the same workspace,
    calls back to back of growing and shrinking contexts, two shapes in turn."""
    pools = [Pool([2000, 64, 700], 2, 16, "bf16", seed=1), Pool([1, 500], 4, 32, "e4m3", seed=2)]
    first = [_attend(p, 2, 1, seed=3)[1:] for p in pools]
    ws = ckv.workspace(pools[0].shape(2), 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    assert ws.numel() >= ckv.workspace_bytes(pools[1].shape(2), 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    for i in range(30):
        for p, want in zip(pools, first):
            full = p.ctx.clone()
            if i % 3 == 1:
                p.ctx.copy_(torch.clamp(full - 100 * i, min=0))
            got = _attend(p, 2, 1, seed=3, ws=ws)[1:]
            if i % 3 == 1:
                p.ctx.copy_(full)
            else:
                assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- debug mode --------------------------------------------------------------------------
@pytest.fixture
def debug_mode():
    ckv.set_debug(True)
    try:
        yield
    finally:
        ckv.set_debug(False)


def test_debug_mode_names_bad_inputs(debug_mode):
    pool = Pool([50, 20], 1, 16, "bf16", holes=[(1, 0)], max_ctx=64)
    s = pool.shape(2)
    q, out, lse = _attend(pool, 2, 1)         # -1 entries are fine
    _check_attention(pool, q, out, lse, 1)
    scores = torch.empty((2, 1, 64), device=DEV)

    def refused(what, call):
        with pytest.raises(ckv.CkvError) as e:
            call()
        assert e.value.status == 1 and what in str(e.value), str(e.value)

    qd = q[:, 0].to(DEV)
    score = lambda: ckv.paged_score_keys(s, pool.cache, qd, pool.ctx, SCALE, scores)  # noqa: E731
    pool.table[0, 1] = pool.k.shape[0]
    refused("page_table[0][1]", score)
    pool.table[0, 1], pool.table[0, 3] = 0, 1 << 20
    pool.ctx[0] = 48                          # the bad entry is past the length
    score()
    pool.ctx[1] = 65
    refused("ctx_lens[1]", score)
    pool.ctx[1] = 20
    k = torch.zeros((1, 1, D), dtype=torch.bfloat16, device=DEV)
    for req, pos, what in ((0, 64, "positions[0]"), (2, 0, "requests[0]"), (1, 3, "no page"),
                           (0, 50, "no page")):
        i32 = lambda v: torch.tensor([v], dtype=torch.int32, device=DEV)  # noqa: E731
        refused(what, lambda: ckv.paged_write(s, pool.cache, i32(req), i32(pos), k, k))
    ckv.paged_write(s, pool.cache, None, torch.tensor([-1], dtype=torch.int32, device=DEV), k, k)
