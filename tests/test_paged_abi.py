"""The rotary positions and the paged cache without a GPU: refusals on the
host, struct mirrors, frequencies against their formulas, and the plain
64-bit forms of the GPU tests against numbers worked out by hand."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2607_26475_amd as ckv
from paged_helpers import e4m3_64, rope64, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ckv.h")
FAKE = 0x100000
STATUS = {"OK": 0, "EINVAL": 1, "ESHAPE": 2, "EUNSUPPORTED": 3, "EWORKSPACE": 4}


def shape(**kw):
    return ckv.shape_for(**dict(dict(batch=2, num_q_heads=8, num_kv_heads=2, max_ctx=64), **kw))


def cache(**kw):
    d = dict(k_pages=FAKE, v_pages=FAKE, k_exps=None, v_exps=None, page_table=FAKE,
             page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128, kind=0,
             page_size=16, num_pages=9, table_stride=4)
    d.update(kw)
    return ckv.PagedCache(*d.values())


def rope(**kw):
    d = dict(inv_freq=FAKE, head_dim=128, rot_dim=128, layout=0, type=0, inverse=0, scale=1.0)
    d.update(kw)
    return ckv.Rope(*d.values())


def rows(**kw):
    d = dict(src=FAKE, dst=FAKE + 4096, st=1024, sh=128, dt=1024, dh=128, heads=8, reserved=0)
    d.update(kw)
    return ckv.Rows(*d.values())


def test_struct_mirrors(tmp_path):
    """The ctypes mirrors have the C compiler's offsets and sizes."""
    structs = {"ckv_rope": ckv.Rope, "ckv_rows": ckv.Rows, "ckv_paged_cache": ckv.PagedCache,
               "ckv_rope_scaling": ckv.RopeScaling}
    lines = []
    for name, s in structs.items():
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in s._fields_]
        lines.append(f'printf("%zu\\n", sizeof({name}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ckv.h"\nint main(void) {\n' +
                   "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    want = []
    for s in structs.values():
        want += [getattr(s, f).offset for f, _ in s._fields_] + [ctypes.sizeof(s)]
    assert got == want


def test_constants_match_the_header():
    text = open(HEADER).read()
    vals = dict(re.findall(r"(CKV_(?:ROPE|CACHE)_\w+) = (\d+)", text))
    assert len(vals) == 11
    for name, v in vals.items():
        assert getattr(ckv, name[4:]) == int(v), name
    total = int(re.search(r"CKV_K_TOTAL = (\d+)", text).group(1))
    assert total == ckv.KERNEL_COUNT == len(ckv.KERNEL_IDS)
    assert [ckv._lib.ckv_kernel_name(i).decode() for i in range(total)] == list(ckv.KERNEL_IDS)
    assert ckv._lib.ckv_kernel_name(total) == b""


def test_kernel_stats_keep_their_size():
    """ckv_profile_end writes the 16 classes it always did."""
    lib, guard = ckv._lib, 7
    arr = (ckv.KernelStats * 17)()
    arr[16].launches = guard
    assert lib.ckv_profile_begin(0xFFFFFFFF) == 0
    assert lib.ckv_profile_end(arr) == 0 and arr[16].launches == guard
    for count in (0, -1, ckv.KERNEL_COUNT + 1):
        assert lib.ckv_profile_end_n(arr, count) == STATUS["EINVAL"]
    assert lib.ckv_profile_end_n(None, 3) == STATUS["EINVAL"]
    assert lib.ckv_profile_end_n(arr, 17) == 0 and arr[16].launches == 0


def call_rope(r=None, n=5, pos=FAKE, q=None, k=None):
    return ckv._lib.ckv_rope_rows(r or rope(), n, pos, q or rows(), k, None)


@pytest.mark.parametrize("kw,status", [
    (dict(inv_freq=None), "EINVAL"), (dict(inv_freq=FAKE + 8), "EINVAL"),
    (dict(head_dim=4, rot_dim=2), "EUNSUPPORTED"), (dict(head_dim=132), "EUNSUPPORTED"),
    (dict(head_dim=2048), "EUNSUPPORTED"), (dict(rot_dim=0), "ESHAPE"),
    (dict(rot_dim=3), "ESHAPE"), (dict(rot_dim=130), "ESHAPE"), (dict(layout=2), "EINVAL"),
    (dict(type=2), "EINVAL"), (dict(inverse=2), "EINVAL"), (dict(scale=math.nan), "EINVAL"),
    (dict(scale=math.inf), "EINVAL")])
def test_rope_refusals(kw, status):
    assert call_rope(rope(**kw)) == STATUS[status]
    assert ckv._lib.ckv_last_error_detail() != b""
    write = ckv._lib.ckv_paged_write(shape(), cache(), 2, None, FAKE, FAKE, FAKE, 256, rope(**kw),
                                     None, None)
    assert write in (STATUS[status], STATUS["EUNSUPPORTED"])


@pytest.mark.parametrize("kw,status", [
    (dict(src=None), "EINVAL"), (dict(dst=None), "EINVAL"), (dict(src=FAKE + 2), "EINVAL"),
    (dict(dst=FAKE + 4104), "EINVAL"), (dict(reserved=1), "EINVAL"), (dict(heads=0), "ESHAPE"),
    (dict(heads=4097), "ESHAPE"), (dict(st=1020), "ESHAPE"), (dict(sh=-128), "ESHAPE"),
    (dict(dt=1 << 40), "ESHAPE"), (dict(dst=FAKE, dt=2048), "EINVAL"), (dict(dh=64), "ESHAPE"),
    (dict(dt=0), "ESHAPE"), (dict(dt=512), "ESHAPE"), (dict(dt=128, dh=128), "ESHAPE"),
    (dict(heads=1, dt=64), "ESHAPE")])
def test_rows_refusals(kw, status):
    assert call_rope(q=rows(**kw)) == STATUS[status]
    assert call_rope(k=rows(**kw)) == STATUS[status]
    assert ckv._lib.ckv_paged_write(shape(), cache(), 2, None, FAKE, FAKE, FAKE, 256, rope(),
                                    rows(**kw), None) == STATUS[status]


def test_rope_call_refusals():
    assert call_rope(n=-1) == STATUS["ESHAPE"]
    assert call_rope(n=(1 << 24) + 1) == STATUS["ESHAPE"]
    assert call_rope(pos=None) == STATUS["EINVAL"]
    assert call_rope(pos=FAKE + 4) == STATUS["EINVAL"]
    assert call_rope(q=rows(heads=4000), k=rows(heads=97)) == STATUS["ESHAPE"]
    assert ckv._lib.ckv_rope_rows(None, 1, FAKE, rows(), None, None) == STATUS["EINVAL"]
    assert ckv._lib.ckv_rope_rows(rope(), 1, FAKE, None, None, None) == STATUS["EINVAL"]
    assert call_rope(n=0) == 0
    # heads outermost; one row for every token and head as the source
    assert call_rope(n=0, q=rows(dt=128, dh=5 * 128, st=0, sh=0)) == 0
    # fp32 rows: strides of 16 bytes are 4 elements
    assert call_rope(rope(type=1), n=0, q=rows(st=1020, dt=1020)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k_pages=None), "EINVAL"), (dict(v_pages=FAKE + 8), "EINVAL"),
    (dict(page_table=None), "EINVAL"), (dict(kind=2), "EINVAL"), (dict(kind=1), "EINVAL"),
    (dict(k_exps=FAKE), "EINVAL"), (dict(kind=1, k_exps=FAKE, v_exps=FAKE + 1), "EINVAL"),
    (dict(page_size=0), "EUNSUPPORTED"), (dict(page_size=24), "EUNSUPPORTED"),
    (dict(page_size=1 << 17), "EUNSUPPORTED"), (dict(num_pages=0), "ESHAPE"),
    (dict(table_stride=3), "ESHAPE"), (dict(row_stride=64), "ESHAPE"),
    (dict(row_stride=132), "ESHAPE"), (dict(head_stride=0), "ESHAPE"),
    (dict(page_stride=1 << 37), "ESHAPE"),
    (dict(kind=1, k_exps=FAKE, v_exps=FAKE, row_stride=136), "ESHAPE"),
    (dict(page_size=65536, row_stride=16384), "EUNSUPPORTED"),
    (dict(page_stride=1 << 36, num_pages=(1 << 31) - 1), "ESHAPE")])
def test_cache_refusals(kw, status):
    """The same ones at every entry that takes a cache."""
    lib, s, c = ckv._lib, shape(), cache(**kw)
    got = [lib.ckv_paged_write(s, c, 2, None, FAKE, FAKE, FAKE, 256, None, None, None),
           lib.ckv_paged_read(s, c, FAKE, None, None, 8, FAKE, FAKE, None),
           lib.ckv_paged_score_keys(s, c, FAKE, FAKE, 0.1, FAKE, None),
           lib.ckv_paged_decode_attn(s, c, 1, FAKE, FAKE, 0.1, FAKE, None, FAKE, 1 << 30, None)]
    assert got == [STATUS[status]] * 4


def test_paged_call_refusals():
    lib, s, c = ckv._lib, shape(), cache()

    def write(n=2, req=None, pos=FAKE, k=FAKE, v=FAKE, stride=256, r=None, q=None, s=s):
        return lib.ckv_paged_write(s, c, n, req, pos, k, v, stride, r, q, None)

    assert write(n=3) == STATUS["ESHAPE"]                    # without requests: one a request
    assert write(n=-1) == STATUS["ESHAPE"]
    assert write(stride=128) == STATUS["ESHAPE"] and write(stride=260) == STATUS["ESHAPE"]
    assert write(req=FAKE + 4) == STATUS["EINVAL"] and write(pos=None) == STATUS["EINVAL"]
    assert write(k=None) == STATUS["EINVAL"] and write(v=FAKE + 2) == STATUS["EINVAL"]
    assert write(q=rows()) == STATUS["EINVAL"]               # q without rope
    assert write(r=rope(type=1)) == STATUS["EUNSUPPORTED"]
    assert write(r=rope(head_dim=64, rot_dim=64)) == STATUS["EUNSUPPORTED"]
    assert write(n=0) == 0 and write(n=0, s=shape(batch=0)) == 0

    def read(lens=FAKE, idx=None, n_sel=None, k=8, kd=FAKE, vd=FAKE):
        return lib.ckv_paged_read(s, c, lens, idx, n_sel, k, kd, vd, None)

    assert read(lens=None) == STATUS["EINVAL"] and read(kd=None) == STATUS["EINVAL"]
    assert read(n_sel=FAKE) == STATUS["EINVAL"] and read(idx=FAKE) == STATUS["EINVAL"]
    assert read(k=0) == STATUS["ESHAPE"] and read(k=(1 << 30) + 1) == STATUS["ESHAPE"]
    assert read(idx=FAKE, n_sel=FAKE, k=(1 << 20) + 1) == STATUS["ESHAPE"]
    assert read(vd=FAKE + 8) == STATUS["EINVAL"]

    def score(s=s, q=FAKE, lens=FAKE, scale=0.1, out=FAKE, c=c):
        return lib.ckv_paged_score_keys(s, c, q, lens, scale, out, None)

    assert score(q=None) == STATUS["EINVAL"] and score(out=FAKE + 4) == STATUS["EINVAL"]
    assert score(scale=0.0) == STATUS["EINVAL"] and score(lens=None) == STATUS["EINVAL"]
    assert score(s=shape(batch=0)) == 0

    need = ckv.workspace_bytes(s, 2, ckv.ENTRY_PAGED_DECODE_ATTN)

    def attn(T=2, q=FAKE, lens=FAKE, scale=0.1, out=FAKE, lse=None, ws=FAKE, size=need, s=s):
        return lib.ckv_paged_decode_attn(s, c, T, q, lens, scale, out, lse, ws, size, None)

    assert attn(T=0) == STATUS["EUNSUPPORTED"] and attn(T=5) == STATUS["EUNSUPPORTED"]
    assert attn(q=None) == STATUS["EINVAL"] and attn(out=FAKE + 8) == STATUS["EINVAL"]
    assert attn(lse=FAKE + 4) == STATUS["EINVAL"] and attn(scale=-1.0) == STATUS["EINVAL"]
    assert attn(lens=None) == STATUS["EINVAL"]
    assert attn(ws=None) == STATUS["EWORKSPACE"] and attn(ws=FAKE + 16) == STATUS["EWORKSPACE"]
    assert attn(size=need - 1) == STATUS["EWORKSPACE"]
    assert attn(s=shape(batch=0)) == 0
    with pytest.raises(ckv.CkvError):
        ckv.workspace_bytes(s, 5, ckv.ENTRY_PAGED_DECODE_ATTN)   # 5 tokens of 4 heads
    assert ckv.workspace_bytes(s, 4, ckv.ENTRY_PAGED_DECODE_ATTN) > need
    # bounded however long the context
    assert ckv.workspace_bytes(shape(batch=64, max_ctx=1 << 20), 4,
                               ckv.ENTRY_PAGED_DECODE_ATTN) < 32 << 20


def test_binding_refuses_what_kernels_would_misread():
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    table = torch.zeros((2, 4), dtype=torch.int32)
    c = ckv.paged_cache_for(k, k, table)
    assert (c.page_stride, c.head_stride, c.row_stride, c.num_pages, c.page_size) == \
        (4096, 2048, 128, 4, 16)
    n = ckv.paged_cache_for(k.transpose(1, 2), k.transpose(1, 2), table)
    assert (n.head_stride, n.row_stride, n.page_size) == (128, 2048, 2)
    codes, exps = k.to(torch.float8_e4m3fn), torch.zeros((4, 2, 16), dtype=torch.uint8)
    assert ckv.paged_cache_for(codes, codes, table, exps, exps).kind == ckv.CACHE_E4M3
    for bad in ((k, k[:2], table), (k, k.float(), table), (k.half(), k.half(), table),
                (k, k, table.long()), (k, k, table, exps, exps), (codes, codes, table),
                (codes, codes, table, exps, exps[:2]), (codes, codes, table, exps, exps.int()),
                (k[..., ::2], k[..., ::2], table)):
        with pytest.raises(ValueError):
            ckv.paged_cache_for(*bad)
    with pytest.raises(ValueError):
        ckv.rope_for(torch.zeros(64))                            # fp32 frequencies
    with pytest.raises(ValueError):
        ckv.rope_for(torch.zeros(16, dtype=torch.float64), rot_dim=64)
    with pytest.raises(ValueError):
        ckv.rows_for(torch.zeros(2, 3, 128), torch.zeros(2, 3, 64))
    r = ckv.rope_for(torch.zeros(64, dtype=torch.float64))
    x = ckv.rows_for(torch.zeros((3, 2, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        ckv.rope_rows(r, torch.zeros(3, dtype=torch.int64), x)
    with pytest.raises(ValueError):
        ckv.rope_rows(r, torch.zeros(4, dtype=torch.int32), x)   # more tokens than rows
    with pytest.raises(ValueError):
        ckv.rope_rows(r, torch.zeros(3, dtype=torch.int32), ckv.rows_for(torch.zeros(3, 2, 128)))
    with pytest.raises(ValueError, match="GPU"):                 # all as it should be, but here
        ckv.rope_rows(r, torch.zeros(3, dtype=torch.int32), x)
    s = shape()
    with pytest.raises(ValueError):                              # 5 pages a request, 4 in the table
        ckv.paged_score_keys(shape(max_ctx=65), c, torch.zeros(2, 8, 128).bfloat16(),
                             torch.zeros(2, dtype=torch.int32), 0.1, torch.zeros(2, 2, 65))
    pos, lens = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    kv = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ckv.paged_write(s, c, None, pos, kv[:1], kv[:1])
    with pytest.raises(ValueError):
        ckv.paged_write(s, c, None, pos, kv.float(), kv.float())
    with pytest.raises(ValueError):
        ckv.paged_write(shape(num_kv_heads=1), c, None, pos, kv, kv)
    with pytest.raises(ValueError):
        ckv.paged_read(s, c, lens, None, None, 9, kv, kv)        # too small
    with pytest.raises(ValueError):
        ckv.paged_score_keys(s, c, torch.zeros(2, 8, 128).bfloat16(), lens[:1], 0.1, kv)
    with pytest.raises(ValueError):
        ckv.paged_decode_attn(s, c, 1, torch.zeros(2, 8, 128).bfloat16(), lens, 0.1,
                              torch.zeros(2, 8, 64), None, None)


# ---- frequencies -----------------------------------------------------------------------
def test_frequencies_follow_their_formulas():
    n, base, L, F = 128, 500000.0, 8192, 8.0
    plain = [base ** (-2 * i / n) for i in range(n // 2)]

    def freq(*a):
        f, s = ckv.rope_frequencies(n, base, *a)
        return f.tolist(), s

    close = lambda a, b: all(abs(x - y) <= 1e-14 * y for x, y in zip(a, b))  # noqa: E731
    assert close(freq()[0], plain) and freq()[1] == 1.0
    assert close(freq(ckv.ROPE_LINEAR, F)[0], [f / F for f in plain])
    based = freq(ckv.ROPE_BASE, F)[0]
    assert based[0] == 1.0 and abs(based[-1] - plain[-1] / F) <= 1e-13 * plain[-1]
    turns = [L * f / (2 * math.pi) for f in plain]
    want = [f if t >= 4 else f / F if t <= 1 else
            f * (t - 1) / 3 + f / F * (1 - (t - 1) / 3) for f, t in zip(plain, turns)]
    assert close(freq(ckv.ROPE_BANDS, F, L, 1.0, 4.0)[0], want)
    # the ramp: whole pairs that make 32 turns at one end, 1 turn at the other
    lo = max(max(i for i in range(n // 2) if turns[i] >= 32), 0)   # floor of the index of 32
    hi = min(min(i for i in range(n // 2) if turns[i] <= 1), n - 1)  # ceiling of that of 1
    want = []
    for i, f in enumerate(plain):
        r = min(max((i - lo) / (hi - lo), 0), 1)
        want.append(f * (1 - r) + f / F * r)
    got, scale = freq(ckv.ROPE_RAMP, F, L, 1.0, 32.0)
    assert close(got, want) and abs(scale - (0.1 * math.log(F) + 1)) < 1e-7
    for kind in (ckv.ROPE_LINEAR, ckv.ROPE_BASE):
        assert close(freq(kind, 1.0)[0], plain)
    assert close(ckv.rope_frequencies(2, 10.0)[0].tolist(), [1.0])


@pytest.mark.parametrize("args,status", [
    ((0, 1e4), "ESHAPE"), ((7, 1e4), "ESHAPE"), ((1026, 1e4), "ESHAPE"), ((64, 1.0), "EINVAL"),
    ((64, math.inf), "EINVAL"), ((64, 1e4, 5), "EINVAL"), ((64, 1e4, 1, 0.5), "EINVAL"),
    ((64, 1e4, 1, math.nan), "EINVAL"), ((2, 1e4, 2, 4.0), "ESHAPE"),
    ((64, 1e4, 3, 8.0, 0, 1.0, 4.0), "EINVAL"), ((64, 1e4, 3, 8.0, 4096, 4.0, 4.0), "EINVAL"),
    ((64, 1e4, 4, 8.0, 4096, 0.0, 32.0), "EINVAL")])
def test_frequency_refusals(args, status):
    with pytest.raises(ckv.CkvError) as e:
        ckv.rope_frequencies(*args)
    assert e.value.status == STATUS[status]


# ---- the plain forms themselves ------------------------------------------------------------
def test_plain_rotation_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    f = torch.tensor([math.pi / 2, math.pi], dtype=torch.float64)
    half = rope64(x, torch.tensor([1]), f, 4, False)[0, 0]
    assert torch.allclose(half, torch.tensor([-3.0, -2.0, 1.0, -4.0, 5.0]).double(), atol=1e-15)
    pairs = rope64(x, torch.tensor([1]), f, 4, True, scale=2.0)[0, 0]
    assert torch.allclose(pairs, torch.tensor([-4.0, 2.0, -6.0, -8.0, 5.0]).double(), atol=1e-14)


def test_plain_e4m3_against_torch():
    """Where no exponent is needed (max 256 .. 448), the codes are those of a
    plain conversion; every finite code stands for itself."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn((64, 128), generator=g) * 60
    x[:, 0] = 448.0
    x = x.clamp(-448, 448)
    codes, e = e4m3_64(x.double())
    assert torch.all(e == 127)
    assert torch.equal(codes, x.to(torch.float8_e4m3fn).view(torch.uint8))
    every = torch.arange(256).to(torch.uint8)
    every = every[(every & 0x7F) != 0x7F]
    v = every.view(torch.float8_e4m3fn).double()[None]
    codes, e = e4m3_64(v * 2.0 ** -30)
    assert torch.equal(codes[0], every) and int(e[0]) == 97
    assert torch.equal(values(codes, e), v * 2.0 ** -30)


def test_no_tokens():
    """Empty tensors have no address; all else is checked as ever."""
    lib, r = ckv._lib, rope()
    none = rows(src=None, dst=None)
    assert lib.ckv_rope_rows(r, 0, None, none, none, None) == 0
    assert lib.ckv_rope_rows(r, 1, FAKE, none, None, None) == STATUS["EINVAL"]
    assert lib.ckv_rope_rows(rope(rot_dim=3), 0, None, none, None, None) == STATUS["ESHAPE"]
    s, c = shape(), cache()
    write = lambda n, stride: lib.ckv_paged_write(  # noqa: E731
        s, c, n, None, None, None, None, stride, r, none, None)
    wide = s.num_kv_heads * 128
    assert write(0, wide) == 0
    assert write(0, wide - 8) == STATUS["ESHAPE"] and write(1, wide) == STATUS["EINVAL"]
