"""Attention over selected blocks at the ends of its types' ranges (MI355X only)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from blocks_helpers import attend64, landmarks64, select64
from paged_helpers import D, SCALE
from test_gpu_blocks import DEV, Call, _i32, _log, make

pytestmark = pytest.mark.gpu


def _put(pool, what, p, value, byte):
    """Position p of request 0 of every head of an e4m3 pool: `value` [D] (multiples of
    codes) with exponent byte `byte`, on the device and in the plain form."""
    code = value.float().to(torch.float8_e4m3fn)
    page = int(pool.table[0, p // pool.page])
    getattr(pool, what)[page, :, p % pool.page] = code.view(torch.uint8).to(DEV)
    getattr(pool, what + "_exps")[page, :, p % pool.page] = byte
    getattr(pool, what.upper())[0, :, p] = code.double() * 2.0 ** (byte - 127)


def test_landmarks_past_the_largest_bf16():
    """Means of e4m3 keys up to 448 * 2^127: to the nearest bf16, infinite from
    halfway past the largest one on, with their signs."""
    block = 32
    pool = make("e4m3", [16 * block], 2, 16, seed=1)
    # 2^127 times: the largest bf16 is 2 - 2^-7, the middle to 2 is 2 - 2^-8
    sums = [(2.0, 32), (2.0, 31), (2.0, 30), (2.0, 29), (1.875, 32), (2.125, 32)]
    for j, (x, m) in enumerate(sums):
        for i in range(block):
            v = torch.full((D,), x if i < m else 1.875, dtype=torch.float64)
            v[::2] = -v[::2]
            v[5] = 0.25
            _put(pool, "k", j * block + i, 128 * v, 247)
    for j, byte in enumerate(range(247, 255), len(sums)):
        for i in range(block):
            v = torch.arange(D, dtype=torch.float64) % 9 - 4
            v[7] = (-1.0) ** byte * (448 if i % 2 else 416)
            _put(pool, "k", j * block + i, v, byte)
    _put(pool, "k", 14 * block + 3, torch.full((D,), math.nan), 254)
    c = Call(pool, 4, block, 5, 1)
    c.landmarks()
    got, want = c.marks.cpu(), landmarks64(pool, block)
    assert torch.isinf(want).sum() > 100 and torch.isnan(want).any()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])
    # and what is selected by them
    q = torch.randn((1, 8, D), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    c.select(_i32([0]), _i32([16 * block - 1]), q.to(DEV))
    assert torch.equal(c.idx.cpu(), select64(pool, block, 5, [0], [16 * block - 1], q, want))


def _rising(pool, block, G, Hkv):
    """Keys along one direction whose logits rise by about 5 (a factor of 2^7.1 of the
    weights) in four blocks, and queries along it."""
    u = torch.ones(D, dtype=torch.float64)
    q = (u / 4).expand(1, G * Hkv, D).to(torch.bfloat16)      # q . u * SCALE = 2.83
    for p in range(pool.lens[0]):
        x = u * (0.4375 * (p // block) + 0.0625 * (p % 4))
        if pool.kind == "e4m3":
            _put(pool, "k", p, x.float().to(torch.float8_e4m3fn).double(), 127)
        else:
            x = x.to(torch.bfloat16)
            pool.k[int(pool.table[0, p // pool.page]), :, p % pool.page] = x.to(DEV)
            pool.K[0, :, p] = x.double()
    return q


@pytest.mark.parametrize("kind,new,Hkv,G", [("e4m3", 1, 1, 16), ("e4m3", 40, 2, 16),
                                            ("bf16", 40, 2, 16), ("bf16", 1030, 2, 16)])
def test_large_values_under_rising_logits(kind, new, Hkv, G):
    """Values far up in their types' ranges, each block's logits a little above the
    one before's: every output is a mean of finite values, and finite."""
    _log("rising", kind, new, Hkv, G)
    block, k = 32, 16
    n = block * k + max(64, new)
    pool = make(kind, [n], Hkv, 16, seed=3)
    q = _rising(pool, block, G, Hkv).expand(new, -1, -1).contiguous()
    g = torch.Generator().manual_seed(4)
    for p in range(n):
        v = (torch.randint(1, 8, (D,), generator=g) - 4).double()
        v[3] = 2.0
        if kind == "e4m3":  # 2^120 and less, as subnormal codes under the largest exponents
            _put(pool, "v", p, v * 2.0 ** -9, 254 - p % 7)
        else:
            v = (v * 2.0 ** 117).to(torch.bfloat16)
            pool.v[int(pool.table[0, p // pool.page]), :, p % pool.page] = v.to(DEV)
            pool.V[0, :, p] = v.double()
    pos = list(range(n - new, n))
    idx = torch.arange(k, dtype=torch.int32).expand(new, Hkv, k).contiguous()
    c = Call(pool, G, block, k, new)
    c.idx.copy_(idx)
    c.attend(_i32([0] * new), _i32(pos), q.to(DEV))
    some = sorted({0, new // 2, new - 1})
    out, lse, tol = attend64(pool, block, [0] * len(some), [pos[i] for i in some], q[some],
                             idx[some])
    got = c.out.cpu().double()[some]
    assert torch.isfinite(got).all()
    err = (got - out).abs().amax(-1)
    assert torch.all(err <= tol), float((err / tol).max())


def _best(marks, q, want):
    """The best of the blocks by exactly rounded sums (in fp64 one after the other, terms
    that cancel may take the others with them), ascending."""
    terms = (marks.double()[:, None] * q.double()).tolist()
    s = [max(math.fsum(h) if all(map(math.isfinite, h)) else
             (lambda x: x if x == x else -math.inf)(sum(h)) for h in b) for b in terms]
    order = sorted((j for j in range(len(s)) if s[j] > -math.inf), key=lambda j: (-s[j], j))
    return sorted(order[:want])


def test_scores_past_fp32():
    """Sums of finite products that pass fp32's range, either way or on the way:
    they rank as what they are."""
    block, nb, k = 32, 40, 9
    n = block * nb
    pool = make("bf16", [n], 1, 16, seed=1)
    g = torch.Generator().manual_seed(8)
    far = torch.randn((nb, D), generator=g).double()
    q = torch.randn((1, 2, D), generator=g).double()
    cases = [(2.0 ** 70 * far, 2.0 ** 70 * q), (-2.0 ** 70 * far.abs(), 2.0 ** 70 * q.abs())]
    cancel, qc = far.clone(), q.clone()      # infinite terms that cancel
    qc[..., :2], cancel[:, 0], cancel[:, 1] = 2.0 ** 80, 2.0 ** 60, -2.0 ** 60
    cases.append((cancel, qc))
    one = far.clone()                        # one head of the two passes it downwards
    one[:, 0] = -2.0 ** 100
    q1 = q.clone()
    q1[0, 0, 0], q1[0, 1, 0] = 2.0 ** 100, 0.0
    cases.append((one, q1))
    gone = 2.0 ** 70 * far                   # and landmarks that are no numbers among them
    gone[3, 5], gone[7, 2] = math.nan, -math.inf
    cases.append((gone, 2.0 ** 70 * q.abs()))
    for kept in (k, 64):
        c = Call(pool, 2, block, kept, 1)
        for i, (m, x) in enumerate(cases):
            _log("case", kept, i)
            marks, x = m[None, None].to(torch.bfloat16), x.to(torch.bfloat16)
            c.marks.copy_(marks)
            c.select(_i32([0]), _i32([n - 1]), x.to(DEV))
            best = _best(marks[0, 0, :nb - 1], x[0], kept - 1) + [nb - 1]
            assert c.idx.flatten().tolist() == best + [-1] * (kept - len(best)), i


@pytest.mark.parametrize("page", [16, 256])
def test_bytes_of_unwritten_rows_cost_nothing(page):
    """Decode tokens early in their own blocks of 256 four-bit positions: exponent
    bytes behind the contexts, NaN's or others, change neither bits nor times."""
    B, Hkv, G, k, block = 64, 8, 16, 20, 256
    n = block * k - block + 5
    pool = make("e2m1", [n], Hkv, page, seed=2, max_ctx=block * k, spare=0)
    table = pool.table.expand(B, -1).contiguous()
    last = n - 1
    end = int(pool.table[0, last // page])
    q = torch.randn((B, G * Hkv, D), generator=torch.Generator().manual_seed(2))
    q = q.to(torch.bfloat16).to(DEV)
    idx = torch.arange(k, dtype=torch.int32, device=DEV).expand(B, Hkv, k).contiguous()
    shape = ckv.shape_for(B, G * Hkv, Hkv, block * k)
    ws = ckv.blocks_workspace(shape, block, k, B)
    pos = _i32([last] * B)
    caches, keep = [], []
    for byte in (127, 255):
        e = pool.v_exps.clone()
        e[end, :, last % page + 1:] = byte
        keep.append(e)
        caches.append(ckv.paged_cache_for(pool.k, pool.v, table, pool.k_exps, e))
    outs = [torch.empty((B, G * Hkv, D), device=DEV) for _ in caches]
    times = [[], []]
    for turn in range(8):
        for i, c in enumerate(caches):
            ckv.profile_begin(["block_attn"])
            for _ in range(10):
                ckv.paged_block_attn(shape, c, block, k, None, pos, q, idx, SCALE, outs[i], None,
                                     ws)
            ran = ckv.profile_end()["block_attn"]
            times[i].append(ran[1] / ran[0])
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0]).all()
    _log("times", [1e3 * min(t) for t in times])
    # (a second pass over the blocks would double it)
    assert min(times[1]) <= 1.3 * min(times[0])
