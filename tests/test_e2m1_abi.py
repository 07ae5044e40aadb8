"""The paged cache in four bits without a GPU: refusals, the binding's handle,
and the plain form that the GPU tests compare with."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_26475_amd as ckv
from e2m1_helpers import GRID, e2m1_64, values4

FAKE = 0x100000
STATUS = {"OK": 0, "EINVAL": 1, "ESHAPE": 2, "EUNSUPPORTED": 3}


def _cache(**kw):
    d = dict(k_pages=FAKE, v_pages=FAKE, k_exps=FAKE, v_exps=FAKE, page_table=FAKE,
             page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128,
             kind=ckv.CACHE_E2M1, page_size=16, num_pages=9, table_stride=4)
    d.update(kw)
    return ckv.PagedCache(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(k_exps=None), "EINVAL"), (dict(v_exps=None), "EINVAL"),
    (dict(v_exps=FAKE + 4), "EINVAL"), (dict(k_pages=FAKE + 8), "EINVAL"),
    (dict(kind=3), "EINVAL"), (dict(row_stride=64), "ESHAPE"),
    (dict(row_stride=144), "ESHAPE"),          # 72 bytes
    (dict(head_stride=2064), "ESHAPE"), (dict(page_stride=4104), "ESHAPE"),
    (dict(page_size=65536, row_stride=65536), "EUNSUPPORTED"), (dict(table_stride=3), "ESHAPE")])
def test_refusals(kw, status):
    lib, c = ckv._lib, _cache(**kw)
    s = ckv.shape_for(2, 8, 2, 64)
    got = [lib.ckv_paged_write(s, c, 2, None, FAKE, FAKE, FAKE, 256, None, None, None),
           lib.ckv_paged_read(s, c, FAKE, None, None, 8, FAKE, FAKE, None),
           lib.ckv_paged_score_keys(s, c, FAKE, FAKE, 0.1, FAKE, None),
           lib.ckv_paged_decode_attn(s, c, 1, FAKE, FAKE, 0.1, FAKE, None, FAKE, 1 << 30, None)]
    assert got == [STATUS[status]] * 4


@pytest.mark.parametrize("kw", [{}, dict(row_stride=160), dict(page_size=65536, row_stride=32768,
                                                                head_stride=1 << 31,
                                                                page_stride=1 << 32)])
def test_empty_calls_pass(kw):
    s, c = ckv.shape_for(0, 8, 2, 64), _cache(**kw)
    lib = ckv._lib
    assert lib.ckv_paged_write(s, c, 0, None, None, None, None, 256, None, None, None) == 0
    assert lib.ckv_paged_read(s, c, FAKE, None, None, 8, FAKE, FAKE, None) == 0
    assert lib.ckv_paged_score_keys(s, c, FAKE, FAKE, 0.1, FAKE, None) == 0
    assert lib.ckv_paged_decode_attn(s, c, 1, FAKE, FAKE, 0.1, FAKE, None, FAKE, 1 << 30,
                                     None) == 0


def test_binding():
    codes = torch.zeros((4, 2, 16, 64), dtype=torch.uint8)
    exps, table = torch.zeros((4, 2, 16, 4), dtype=torch.uint8), torch.zeros((2, 4),
                                                                             dtype=torch.int32)
    c = ckv.paged_cache_for(codes, codes, table, exps, exps)
    assert (c.kind, c.page_stride, c.head_stride, c.row_stride, c.num_pages, c.page_size) == \
        (ckv.CACHE_E2M1, 4096, 2048, 128, 4, 16)
    n = ckv.paged_cache_for(codes.transpose(1, 2), codes.transpose(1, 2), table,
                            torch.zeros((4, 16, 2, 4), dtype=torch.uint8),
                            torch.zeros((4, 16, 2, 4), dtype=torch.uint8))
    assert (n.head_stride, n.row_stride, n.page_size) == (128, 2048, 2)
    if hasattr(torch, "float4_e2m1fn_x2"):
        x2 = codes.view(torch.float4_e2m1fn_x2)
        assert ckv.paged_cache_for(x2, x2, table, exps, exps).kind == ckv.CACHE_E2M1
    one = torch.zeros((1, 1, 1, 64), dtype=torch.uint8)
    c = ckv.paged_cache_for(one, one, table, exps[:1, :1, :1].contiguous(),
                            exps[:1, :1, :1].contiguous())
    assert min(c.page_stride, c.head_stride, c.row_stride) >= 128
    for bad in ((codes, codes, table), (codes, codes, table, exps[..., 0], exps[..., 0]),
                (codes, codes, table, exps, exps[:2]), (codes, codes, table, exps, exps.int()),
                (codes.int(), codes.int(), table, exps, exps),
                (codes.to(torch.bfloat16), codes.to(torch.bfloat16), table),
                (codes[..., :32], codes[..., :32], table, exps, exps)):
        with pytest.raises(ValueError):
            ckv.paged_cache_for(*bad)


def test_plain_form():
    """Against closed values: ties, the border of the exponent, the bounds."""
    x = torch.zeros((1, 128), dtype=torch.float64)
    x[0, :8] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x[0, 32:34] = torch.tensor([6.0 + 2.0 ** -20, -1.0])
    x[0, 64], x[0, 65] = math.inf, 1.0
    x[0, 96], x[0, 97] = 2.0 ** 127.9, 2.0 ** 125
    codes, exps = e2m1_64(x)
    assert exps[0].tolist() == [127, 128, 255, 252]
    v = values4(codes, exps)[0]
    assert v[:8].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert v[32:34].tolist() == [6.0, -1.0]
    assert torch.isnan(v[64:96]).all()
    assert v[96:98].tolist() == [6 * 2.0 ** 125, 2.0 ** 125]
    # every value of the format is its own nearest, and -0 stays
    y = torch.cat([GRID, -GRID]).repeat(8)[None]
    codes, exps = e2m1_64(y)
    assert torch.equal(values4(codes, exps), y)
    assert torch.equal(torch.signbit(values4(codes, exps)), torch.signbit(y))
