"""Attention over selected blocks without a GPU: refusals, workspaces, the binding."""
from __future__ import annotations

import pytest
import torch

import paper_2607_26475_amd as ckv

FAKE = 0x100000
STATUS = {"OK": 0, "EINVAL": 1, "ESHAPE": 2, "EUNSUPPORTED": 3, "EWORKSPACE": 4}
BIG = 1 << 40


def _cache(**kw):
    d = dict(k_pages=FAKE, v_pages=FAKE, k_exps=None, v_exps=None, page_table=FAKE,
             page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128, kind=0,
             page_size=16, num_pages=9, table_stride=4)
    d.update(kw)
    return ckv.PagedCache(*d.values())


def marks(s=None, c=None, block=32, ctx=FAKE, first=FAKE, lm=FAKE):
    return ckv._lib.ckv_paged_landmarks(s or ckv.shape_for(2, 8, 2, 64), c or _cache(), block, ctx,
                                        first, lm, None)


def select(s=None, c=None, block=32, k=4, n=3, req=FAKE, pos=FAKE, q=FAKE, lm=FAKE, idx=FAKE,
           ws=FAKE, size=BIG):
    return ckv._lib.ckv_select_blocks(s or ckv.shape_for(2, 8, 2, 64), c or _cache(), block, k, n,
                                      req, pos, q, lm, idx, ws, size, None)


def attend(s=None, c=None, block=32, k=4, n=3, req=FAKE, pos=FAKE, q=FAKE, idx=FAKE, scale=0.1,
           out=FAKE, lse=FAKE, ws=FAKE, size=BIG):
    return ckv._lib.ckv_paged_block_attn(s or ckv.shape_for(2, 8, 2, 64), c or _cache(), block, k,
                                         n, req, pos, q, idx, scale, out, lse, ws, size, None)


@pytest.mark.parametrize("block", [0, 1, 16, 48, 512, -32])
def test_blocks_of_other_sizes(block):
    assert [marks(block=block), select(block=block), attend(block=block)] == [3] * 3
    with pytest.raises(ckv.CkvError):
        ckv.blocks_workspace_bytes(ckv.shape_for(2, 8, 2, 64), block, 4, 3)


@pytest.mark.parametrize("kw,status", [
    (dict(page_size=8, table_stride=8), "EUNSUPPORTED"), (dict(kind=2), "EINVAL"),
    (dict(table_stride=3), "ESHAPE"), (dict(k_pages=None), "EINVAL")])
def test_caches(kw, status):
    c = _cache(**kw)
    assert [marks(c=c), select(c=c), attend(c=c)] == [STATUS[status]] * 3


def test_calls():
    for f in (select, attend):
        assert f(k=0) == f(k=65) == STATUS["ESHAPE"]
        assert f(n=-1) == f(n=(1 << 24) + 1) == STATUS["ESHAPE"]
        assert f(req=FAKE + 4) == f(pos=None) == f(q=FAKE + 2) == f(idx=None) == STATUS["EINVAL"]
        assert f(req=None, n=3) == STATUS["ESHAPE"]        # three tokens of two requests
        assert f(ws=None) == f(ws=FAKE + 16) == STATUS["EWORKSPACE"]
        need = ckv.blocks_workspace_bytes(ckv.shape_for(2, 8, 2, 64), 32, 4, 3)
        assert f(size=need - 1) == STATUS["EWORKSPACE"]
        # nothing to do: addresses may be NULL
        assert f(n=0, req=None, pos=None, q=None, idx=None, ws=None, size=0) == 0
        s = ckv.shape_for(1, 8, 8, 64)
        assert f(s=s, n=1 << 24) == STATUS["EUNSUPPORTED"]
        assert f(s=ckv.shape_for(2, 24, 8, 64)) == STATUS["EUNSUPPORTED"]
    assert select(lm=None) == STATUS["EINVAL"] and attend(out=FAKE + 8) == STATUS["EINVAL"]
    assert attend(lse=FAKE + 4) == STATUS["EINVAL"]
    for scale in (0.0, -1.0, float("inf"), float("nan"), 2.0 ** 127):
        assert attend(scale=scale) == STATUS["EINVAL"]
    assert marks(ctx=None) == marks(first=FAKE + 4) == marks(lm=FAKE + 8) == STATUS["EINVAL"]
    assert marks(s=ckv.shape_for(0, 8, 2, 64)) == 0
    # more scoring workgroups than a launch may have
    s = ckv.shape_for(1, 16, 1, 1 << 30)
    c = _cache(page_size=65536, row_stride=128, head_stride=65536 * 128, page_stride=65536 * 128,
               table_stride=1 << 14)
    assert select(s=s, c=c, n=1 << 20) == STATUS["EUNSUPPORTED"]


def test_workspace():
    s = ckv.shape_for(16, 32, 8, 65536)
    # 4 bytes a token, head and block, and little more
    n = 4 * 160 * 8 * 1024
    assert n <= ckv.blocks_workspace_bytes(s, 64, 32, 160) <= n + (64 << 10)
    # partial sums of few tokens are bounded
    assert ckv.blocks_workspace_bytes(ckv.shape_for(1, 16, 1, 4096), 256, 16, 1) <= 4.2 * 2 ** 20
    assert ckv.blocks_workspace_bytes(s, 64, 32, 0) == 0


def test_binding_refuses_what_kernels_would_misread():
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    table = torch.zeros((2, 4), dtype=torch.int32)
    c, s = ckv.paged_cache_for(k, k, table), ckv.shape_for(2, 8, 2, 64)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)           # noqa: E731
    q, lm = torch.zeros((3, 8, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 2, 128),
                                                                        dtype=torch.bfloat16)
    out, lse, ws = torch.zeros((3, 8, 128)), torch.zeros((3, 8)), torch.zeros(1 << 20,
                                                                              dtype=torch.uint8)

    def refused(f, *a, **kw):
        with pytest.raises(ValueError) as e:
            f(*a, **kw)
        return "on a GPU" not in str(e.value)

    good = (s, c, 32, 4, i32(3), i32(3), q, lm, i32(3, 2, 4), ws)
    assert not refused(ckv.select_blocks, *good)                 # only the device is missing
    for i, bad in ((4, i32(2)), (5, i32(3).long()), (6, q[:2]), (6, q.float()), (7, lm[:1]),
                   (8, i32(3, 2, 3)), (9, ws.int()), (0, ckv.shape_for(2, 8, 4, 64)),
                   (0, ckv.shape_for(2, 8, 2, 65))):
        assert refused(ckv.select_blocks, *good[:i], bad, *good[i + 1:]), i
    good = (s, c, 32, 4, i32(3), i32(3), q, i32(3, 2, 4), 0.1, out, lse, ws)
    assert not refused(ckv.paged_block_attn, *good)
    assert not refused(ckv.paged_block_attn, *good[:10], None, ws)
    for i, bad in ((6, q[:, :7]), (7, i32(2, 2, 4)), (9, out[:2]), (9, out.bfloat16()),
                   (10, lse[:, :7])):
        assert refused(ckv.paged_block_attn, *good[:i], bad, *good[i + 1:]), i
    assert not refused(ckv.paged_landmarks, s, c, 32, i32(2), lm, first=i32(2))
    for a, kw in (((s, c, 32, i32(1), lm), {}), ((s, c, 32, i32(2), lm[:, :1]), {}),
                  ((s, c, 32, i32(2), lm.float()), {}), ((s, c, 32, i32(2), lm),
                                                         {"first": i32(1)})):
        assert refused(ckv.paged_landmarks, *a, **kw)
