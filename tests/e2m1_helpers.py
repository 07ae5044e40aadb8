"""Plain 64-bit forms of the 4-bit cache (CPU) and pools of its pages for the GPU
tests."""
from __future__ import annotations

import torch

import paper_2607_26475_amd as ckv
from paged_helpers import D, Pool

GROUP = 32
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def e2m1_64(rows):
    """fp64 rows [..., 128] -> (bytes of two codes [..., 64], exponent bytes
    [..., 4]): for 32 elements the smallest e in [-125, 125] with max |x| <= 6 *
    2^e (125 beyond), the nearest codes, ties to the even one, 6 at most; 255
    where one of the 32 is not finite (codes 0 here)."""
    y = rows.unflatten(-1, (-1, GROUP))
    fin = torch.isfinite(y).all(-1)
    y = torch.where(fin[..., None], y, 0)
    most = y.abs().amax(-1)
    m, e = torch.frexp(most)
    e = torch.where(most == 0, -125, torch.where(m <= 0.75, e - 3, e - 2)).clamp(-125, 125)
    z = torch.ldexp(y, -e[..., None])
    dist = (z.abs()[..., None] - GRID).abs()
    near = dist.amin(-1, keepdim=True)
    # of two codes at one distance the even one
    rank = (dist == near).to(torch.int64) * (2 - torch.arange(8) % 2)
    code = rank.argmax(-1) | torch.signbit(y).long() << 3
    code = code.flatten(-2)
    exps = torch.where(fin, e + 127, 255)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), exps.to(torch.uint8)


def values4(codes, exps):
    """What bytes of two codes and exponent bytes stand for, fp64."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    x = GRID[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    s = torch.where(exps == 255, float("nan"), torch.exp2(exps.double() - 127))
    return (x.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


class Pool4(Pool):
    """A pool of e2m1 pages: rows that nobody may read have NaN exponents."""

    def __init__(self, lens, Hkv, page, seed=0, order="heads", holes=(), spare=2, max_ctx=None,
                 share=False):
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
        shape = (P, Hkv, page, D // 2)
        k, v = (torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) for _ in "kv")
        ke, ve = (torch.randint(123, 129, (P, Hkv, page, 4), generator=g, dtype=torch.uint8)
                  for _ in "kv")
        kd, vd = values4(k, ke), values4(v, ve)
        pos = torch.arange(self.max_ctx)
        pg = table[:, pos // page].long()
        self.there = (pg >= 0) & (pos < torch.tensor(self.lens)[:, None])
        at = (pg.clamp(min=0), slice(None), (pos % page).expand(B, -1))
        self.K = kd[at].transpose(1, 2).contiguous()
        self.V = vd[at].transpose(1, 2).contiguous()
        used = torch.zeros((P, page), dtype=torch.bool)
        bb, pp = torch.nonzero(self.there, as_tuple=True)
        used[pg[bb, pp], pp % page] = True
        bad = ~used[:, None].expand(P, Hkv, page)
        ke[bad], ve[bad] = 255, 255
        self.k_exps, self.v_exps = ke.to(dev), ve.to(dev)
        if order == "heads":
            self.k, self.v = k.to(dev), v.to(dev)
        elif order == "rows":
            self.k = k.transpose(1, 2).contiguous().to(dev).transpose(1, 2)
            self.v = v.transpose(1, 2).contiguous().to(dev).transpose(1, 2)
        else:
            kv = torch.stack([k, v], 3).to(dev)  # [P][H][page][2][64]
            self.k, self.v = kv[:, :, :, 0], kv[:, :, :, 1]
        self.table = table.to(dev)
        self.page, self.kind, self.Hkv, self.B = page, "e2m1", Hkv, B
        self.ctx = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.cache = ckv.paged_cache_for(self.k, self.v, self.table, self.k_exps, self.v_exps)
