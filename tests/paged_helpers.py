"""Plain 64-bit forms of the rotary positions and the paged cache (CPU), and
pools of pages for their GPU tests."""
from __future__ import annotations

import math

import torch

import paper_2607_26475_amd as ckv

D = 128
SCALE = 0.08838834764831845
U24 = 2.0 ** -24                 # half a step of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U24}
# Relative to |x1| + |x2|, in halves of an fp32 step: the reduced angle (its
# rounding, the constant's and the product's, at most pi/4 of a radian: under 3),
# the series' sums (2), the scale (1), the two products and their sum (2)
ROPE_HALVES = 8


def rope64(x, pos, inv_freq, rot, interleaved, inverse=False, scale=1.0):
    """x [N][heads][d] (any type) -> fp64 rotated rows."""
    y = x.double().clone()
    a = pos.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(a) * scale, torch.sin(a) * (-scale if inverse else scale)
    i1 = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    i2 = i1 + 1 if interleaved else i1 + rot // 2
    x1, x2 = x.double()[..., i1], x.double()[..., i2]
    y[..., i1], y[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def rope_slack(x, rot, interleaved, scale=1.0):
    """The fp32 part of a rotation's error, element by element."""
    m = torch.zeros_like(x, dtype=torch.float64)
    i1 = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    i2 = i1 + 1 if interleaved else i1 + rot // 2
    both = (x.double()[..., i1].abs() + x.double()[..., i2].abs()) * abs(scale)
    m[..., i1], m[..., i2] = both, both
    return ROPE_HALVES * U24 * m


def e4m3_64(rows):
    """fp64 rows [..., d] -> (codes as uint8, exponent bytes as uint8): the
    smallest e in [-127, 127] with max finite |x| <= 448 * 2^e, nearest codes,
    ties to even; infinities and NaN as NaN."""
    fin = torch.isfinite(rows)
    most = torch.where(fin, rows.abs(), 0).amax(-1)
    m, x = torch.frexp(most)
    e = torch.where(most == 0, -127, x - torch.where(m <= 0.875, 9, 8)).clamp(-127, 127)
    y = torch.where(fin, torch.ldexp(rows, -e[..., None]), 0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    val = torch.round(y / step) * step
    code = val.float().to(torch.float8_e4m3fn).view(torch.uint8)  # exact: val is a code's value
    code = torch.where((y < 0) | ((y == 0) & torch.signbit(rows)), code | 0x80, code)
    return torch.where(fin, code, 0x7F).to(torch.uint8), (e + 127).to(torch.uint8)


def values(codes, exps):
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127)[..., None]


class Pool:
    """A paged cache on the device with its rows known on the host: dense fp64
    K, V [B][Hkv][max_ctx][D], whether each position is there, and NaN in every
    row that nobody may read."""

    ORDERS = ("heads", "rows", "pairs")  # [page][head][row], [page][row][head], K|V interleaved

    def __init__(self, lens, Hkv, page, kind, seed=0, order="heads", holes=(), spare=2,
                 max_ctx=None, share=False, rows=None):
        g = torch.Generator().manual_seed(seed)
        dev = torch.device("cuda:0")
        self.lens = list(lens)
        B = len(self.lens)
        self.max_ctx = max_ctx or max(1, max(self.lens))
        per = -(-self.max_ctx // page)
        table = torch.full((B, per), -1, dtype=torch.int32)
        want = [(b, s) for b, n in enumerate(self.lens) for s in range(-(-n // page))
                if (b, s) not in set(holes)]
        perm = torch.randperm(len(want) + spare, generator=g)
        for i, (b, s) in enumerate(want):
            table[b, s] = int(perm[i])
        if share:  # request 1 begins with request 0's first page
            table[1, 0] = table[0, 0]
        P = len(want) + spare
        k = torch.randn((P, Hkv, page, D), generator=g) * torch.exp(
            0.5 * torch.randn((1, Hkv, 1, D), generator=g))
        v = torch.randn((P, Hkv, page, D), generator=g)
        self.k_exps = self.v_exps = None
        if kind == "bf16":
            k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
            kd, vd = k.double(), v.double()
        else:
            r = torch.exp2(torch.randint(-3, 4, (P, Hkv, page, 1), generator=g).double())
            (k, ke), (v, ve) = e4m3_64(k.double() * r), e4m3_64(v.double() / r)
            kd, vd = values(k, ke), values(v, ve)
        # what each request's positions hold, and which positions are there
        pos = torch.arange(rows or self.max_ctx)   # (of long tables only the first)
        pg = table[:, pos // page].long()
        self.there = (pg >= 0) & (pos < torch.tensor(self.lens)[:, None])
        at = (pg.clamp(min=0), slice(None), (pos % page).expand(B, -1))
        self.K = kd[at].transpose(1, 2).contiguous()
        self.V = vd[at].transpose(1, 2).contiguous()
        # rows that nobody may read: NaN
        used = torch.zeros((P, page), dtype=torch.bool)
        bb, pp = torch.nonzero(self.there, as_tuple=True)
        used[pg[bb, pp], pp % page] = True
        bad = ~used[:, None].expand(P, Hkv, page)
        if kind == "bf16":
            k[bad], v[bad] = float("nan"), float("nan")
        else:
            k[bad], v[bad], ke[bad], ve[bad] = 0x7F, 0x7F, 255, 255
            self.k_exps, self.v_exps = ke.to(dev), ve.to(dev)
        if order == "heads":
            self.k, self.v = k.to(dev), v.to(dev)
        elif order == "rows":
            self.k = k.transpose(1, 2).contiguous().to(dev).transpose(1, 2)
            self.v = v.transpose(1, 2).contiguous().to(dev).transpose(1, 2)
        else:
            kv = torch.stack([k, v], 3).to(dev)  # [P][H][page][2][D]
            self.k, self.v = kv[:, :, :, 0], kv[:, :, :, 1]
        self.table = table.to(dev)
        self.page, self.kind, self.Hkv, self.B = page, kind, Hkv, B
        self.ctx = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.cache = ckv.paged_cache_for(self.k, self.v, self.table, self.k_exps, self.v_exps)

    def shape(self, G):
        return ckv.shape_for(self.B, G * self.Hkv, self.Hkv, self.max_ctx)

    def attention(self, q, T):
        """fp64 out, lse and the error that fp32 may have, for q [B][T][Hq][D]."""
        B, H = self.B, self.Hkv
        G = q.shape[2] // H
        out = torch.zeros(q.shape, dtype=torch.float64)
        lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64)
        tol = torch.zeros(q.shape[:3], dtype=torch.float64)
        for b in range(B):
            for t in range(T):
                n = self.lens[b] - (T - 1 - t)
                ok = self.there[b] & (torch.arange(self.there.shape[1]) < n)
                if not ok.any():
                    continue
                for h in range(H):
                    k, v = self.K[b, h, ok], self.V[b, h, ok]
                    x = q[b, t, h * G:(h + 1) * G].double()
                    l = x @ k.T * SCALE
                    out[b, t, h * G:(h + 1) * G] = torch.softmax(l, -1) @ v
                    lse[b, t, h * G:(h + 1) * G] = torch.logsumexp(l, -1)
                    # logits: 128 fp32 sums and the scaling, then weights by them
                    # (the maximum's own error cancels against the sum's); each
                    # of the m positions is one fp32 sum of values up to max |V|
                    d = 130 * U24 * (x.abs() @ k.abs().T).amax(-1) * SCALE
                    m = int(ok.sum())
                    tol[b, t, h * G:(h + 1) * G] = (2 * d + (m + 64) * U24) * v.abs().max()
        return out, lse, tol
