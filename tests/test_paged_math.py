"""The index arithmetic of the paged cache's kernels (no GPU)."""
from __future__ import annotations

import ctypes

import os
import subprocess
import sys

import numpy as np
import pytest

from native_paged import HERE, lib


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 16, 100, 128, 129, 300, 400, 1000])
def test_loaded_halves_stay_in_their_pages(page, n):
    """Every half whose rows a wave loads begins at a multiple of 16 and ends in
    its page and its context, whatever is evicted and wherever a piece ends: the
    whole context, every short piece of it, evicted tails of pieces."""
    so, shift = lib(), page.bit_length() - 1
    rng = np.random.default_rng(page + n)
    slots, steps = -(-n // page), -(-n // 128)
    tables = [np.ones(slots), np.zeros(slots)]
    tables += [np.arange(slots) < i for i in range(slots)]     # a tail evicted
    tables += [rng.random(slots) < q for q in (0.1, 0.5, 0.9) for _ in range(4)]
    first = (ctypes.c_int32 * 64)()
    for there in tables:
        there = np.ascontiguousarray(there, dtype=np.uint8)
        for take in {1, 2, 3, 4, 8, steps}:
            for step in range(steps):
                for wave in range(4):
                    m = so.t_attn_halves(n, shift, there.ctypes.data_as(ctypes.c_void_p), step,
                                         take, wave, first, 64)
                    assert m < 64
                    for f in first[:m]:
                        last = f + so.t_half_last(f, n)
                        assert f % 16 == 0 and 0 <= f <= last < n, (f, last)
                        assert f // page == last // page, (f, last)


def check_table(lens, max_ctx, page, wide, col, num_pages=8):
    """Debug mode's finding about columns col .. of `wide`: None or (kind, request,
    entry)."""
    lens, wide = np.asarray(lens, np.int32), np.ascontiguousarray(wide, np.int32)
    slots = ctypes.c_int()
    got = lib().t_check_table(len(lens), max_ctx, page.bit_length() - 1, num_pages,
                              lens.ctypes.data_as(ctypes.c_void_p),
                              wide.ctypes.data_as(ctypes.c_void_p), wide.shape[1], col,
                              ctypes.byref(slots))
    if got == 2 ** 64 - 1:
        return None
    item = got & (2 ** 56 - 1)
    return got >> 56, item // slots.value, item % slots.value


def test_checked_table_entries_belong_to_positions():
    """Columns of a wider table whose last row ends where memory ends: no entry
    past the columns is read, and only those of positions are judged."""
    code = ("import numpy as np, test_paged_math as t\n"
            "w = np.full((3, 11), 99); w[:, 6:] = 3\n"
            "assert t.check_table([80, 0, 65], 80, 16, w, 6) is None\n"
            "w[2, 8] = 8\n"
            "assert t.check_table([80, 0, 65], 80, 16, w, 6) == (4, 2, 2)\n"
            "assert t.check_table([80, 0, 32], 80, 16, w, 6) is None\n"
            "w[0, 10] = -2\n"
            "assert t.check_table([80, 0, 65], 80, 16, w, 6) == (4, 0, 4)\n"
            "assert t.check_table([64, -5, 32], 80, 16, w, 6) is None\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=HERE, capture_output=True, text=True,
                       env=dict(os.environ, PYTHONPATH=os.path.dirname(HERE)), timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])


def test_debug_flags_are_held_by_one_call():
    flags = ctypes.c_int()
    assert lib().t_flag_pool(8, 2000, ctypes.byref(flags)) == 0
    assert 1 <= flags.value <= 8


@pytest.mark.parametrize("limit", [0, 1, 2, 4])
def test_hand_over_leaves_no_flag(limit):
    """Every order of the two sides' accesses, the wait given up before, between and
    after the other's: what is taken has been given, and the flag is zero again, so
    that the same tag's next launch does not take what is not there yet."""
    so, tag = lib(), 0x9E3779B161C8864E
    outcomes = set()
    for start in (0, 0xFFFFFFFFFFFFFFFF, 12345):
        for turns in range(1 << (limit + 4)):
            word = ctypes.c_uint64(start)
            for replay in range(2):
                got = so.t_hand_over(ctypes.byref(word), tag, limit, turns)
                outcomes.add(got)
                assert word.value == 0, (start, turns, replay)
                assert got != 1, (start, turns, replay)      # taken and not given
    assert {0, 3} <= outcomes <= {0, 2, 3}
