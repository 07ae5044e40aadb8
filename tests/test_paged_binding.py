"""The paged cache's binding without a GPU: what it passes on, and scales."""
from __future__ import annotations

import shutil
import subprocess

import pytest
import torch

import paper_2607_26475_amd as ckv


def _write(n, heads, k, v):
    """A call that all checks of the binding pass ends at the missing GPU."""
    pages = torch.zeros((4, heads, 16, 128), dtype=torch.bfloat16)
    table = torch.zeros((2, 4), dtype=torch.int32)
    ckv.paged_write(ckv.shape_for(2, 4 * heads, heads, 64), ckv.paged_cache_for(pages, pages, table),
                    None, torch.zeros(n, dtype=torch.int32), k, v)


def test_write_takes_single_tokens_and_heads_of_any_stride():
    """K and V of one token from tensors of unlike rows, and heads of one row: the
    strides of a single entry do not matter; all others have to be alike."""
    x, y = (torch.zeros((2, m, 128), dtype=torch.bfloat16) for m in (6, 9))
    for n, heads, k, v in ((1, 2, x[:1, :2], y[:1, 3:5]), (2, 1, x[:, :1], x[:, 3:4]),
                           (2, 1, x[:, :1], x.view(2, 3, 2, 128)[:, 1, ::2]),
                           (2, 2, x[:, :2], x[:, 4:])):
        with pytest.raises(ValueError, match="on a GPU"):
            _write(n, heads, k, v)
    for n, heads, k, v in ((2, 2, x[:, :2], y[:, :2]), (1, 2, x[:1, :2], x[:1, ::3]),
                           (1, 2, x[:1, ::3], x[:1, :2]), (2, 1, x[:, :1], y[:, :1])):
        with pytest.raises(ValueError, match="token stride"):
            _write(n, heads, k, v)


def test_attention_refuses_scales_whose_factor_overflows():
    """A logit of 0 times an infinite factor would be a NaN."""
    fake, s = 0x100000, ckv.shape_for(0, 8, 2, 64)
    c = ckv.PagedCache(fake, fake, None, None, fake, 4096, 2048, 128, 0, 16, 9, 4)
    need = ckv.workspace_bytes(s, 1, ckv.ENTRY_PAGED_DECODE_ATTN)
    for scale, status in ((2.0 ** 126, 0), (1e-30, 0), (2.0 ** 126 * 1.0000002, 1), (2.5e38, 1)):
        assert ckv._lib.ckv_paged_decode_attn(s, c, 1, fake, fake, scale, fake, None, fake, need,
                                              None) == status, scale


def test_a_library_without_an_entry_is_refused_by_name(tmp_path, monkeypatch):
    """An older build of the same ABI version: the first entry it lacks is named."""
    src, so = tmp_path / "old.c", tmp_path / "libold.so"
    names = [n for n in ckv.EXPORTS if "rope" not in n and "paged" not in n]
    src.write_text("int ckv_abi_version(void) { return 9; }\n" + "".join(
        f"int {n}(void) {{ return 0; }}\n" for n in names if n != "ckv_abi_version"))
    subprocess.run([shutil.which("gcc"), "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    monkeypatch.setattr(ckv, "LIB_PATH", str(so))
    with pytest.raises(ImportError, match="ckv_(rope|paged)_"):
        ckv._load()
