"""Plain 64-bit forms of the attention over selected blocks (CPU)."""
from __future__ import annotations

import math

import torch

from paged_helpers import D, SCALE, U24


def landmarks64(pool, block, first=None, old=None):
    """Means of the keys that are there, [B][Hkv][nb][D] as bf16; blocks without
    any, or before first's, as in `old`."""
    nb = -(-pool.max_ctx // block)
    out = torch.zeros((pool.B, pool.Hkv, nb, D), dtype=torch.bfloat16) if old is None else old.clone()
    for b in range(pool.B):
        for j in range((first[b] if first else 0) // block, nb):
            at = torch.arange(j * block, min((j + 1) * block, pool.max_ctx))
            at = at[pool.there[b, at]]
            if len(at):
                out[b, :, j] = pool.K[b][:, at].mean(1).to(torch.bfloat16)
    return out


def block_there(pool, block):
    nb = -(-pool.max_ctx // block)
    t = (pool.table.cpu() >= 0).repeat_interleave(pool.page, 1)[:, :pool.max_ctx]
    t = torch.nn.functional.pad(t, (0, nb * block - pool.max_ctx))
    return t.view(pool.B, nb, block).any(-1)


def select64(pool, block, k, req, pos, q, marks):
    """[N][Hkv][k] int32: own block and the best earlier ones, ascending, -1 padded."""
    N, H = len(req), pool.Hkv
    there = block_there(pool, block)
    out = torch.full((N, H, k), -1, dtype=torch.int32)
    for t, (b, p) in enumerate(zip(req, pos)):
        if not (0 <= p < pool.max_ctx and 0 <= b < pool.B):
            continue
        o = p // block
        for h in range(H):
            x = q[t].double().view(H, -1, D)[h]
            s = (marks[b, h, :o].double() @ x.T).amax(-1)
            s[~there[b, :o] | torch.isnan(s)] = -math.inf
            order = torch.sort(s, descending=True, stable=True).indices[:k - 1]
            order = order[s[order] > -math.inf]
            keep = sorted(order.tolist()) + [o]
            out[t, h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    return out


def attend64(pool, block, req, pos, q, idx):
    """fp64 out, lse and the error that fp32 may have."""
    N, H = len(req), pool.Hkv
    G = q.shape[1] // H
    out = torch.zeros((N, H * G, D), dtype=torch.float64)
    lse = torch.full((N, H * G), -math.inf, dtype=torch.float64)
    tol = torch.zeros((N, H * G), dtype=torch.float64)
    for t, (b, p) in enumerate(zip(req, pos)):
        if not (0 <= p < pool.max_ctx and 0 <= b < pool.B):
            continue
        for h in range(H):
            at = torch.arange(p + 1)
            keep = torch.isin(at // block, idx[t, h][idx[t, h] >= 0].long())
            at = at[keep & pool.there[b, :p + 1]]
            if not len(at):
                continue
            K, V = pool.K[b, h, at], pool.V[b, h, at]
            x = q[t, h * G:(h + 1) * G].double()
            l = x @ K.T * SCALE
            rows = slice(h * G, (h + 1) * G)
            out[t, rows] = torch.softmax(l, -1) @ V
            lse[t, rows] = torch.logsumexp(l, -1)
            # as of the decode attention: logits by 128 fp32 sums and the scaling,
            # m positions one fp32 sum of values up to max |V|
            d = 130 * U24 * (x.abs() @ K.abs().T).amax(-1) * SCALE
            tol[t, rows] = (2 * d + (len(at) + 64) * U24) * V.abs().max()
    return out, lse, tol


def poison(pool, b, h, p, what, value=float("nan")):
    """Makes a row of K or V (``what``) no numbers, on the device and in the plain form."""
    page = int(pool.table[b, p // pool.page])
    at = (page, h, p % pool.page)
    if pool.kind == "bf16":
        getattr(pool, what)[at] = value
    elif pool.kind == "e4m3":
        value = float("nan")                     # its codes have no infinities
        getattr(pool, what)[at] = 0x7F
    else:
        value = float("nan")
        getattr(pool, what + "_exps")[at] = 255
    getattr(pool, what.upper())[b, h, p] = value
