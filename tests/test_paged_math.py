"""The index arithmetic of the paged cache's kernels (no GPU)."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

from native_paged import lib


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
