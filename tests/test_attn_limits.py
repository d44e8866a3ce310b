"""The full-attention layers' format and sizes at their limits, on the CPU."""
import ctypes

import numpy as np
import pytest

from oracle import attention as A
from paper_2608_11231_amd import lkv


def test_largest_rows_of_the_e4m3_oracle():
    """At the largest scale a magnitude stops at 240 * 2^120; below it, and where nothing is that large, rows
    are rounded as ever."""
    top = 255 * 2.0 ** 120  # bf16's largest
    x = np.array([[top, -top, 1.0], [247 * 2.0 ** 120, 248 * 2.0 ** 120, -np.inf], [2.0 ** 127, 225 * 2.0 ** 119, 0.0]])
    codes, byte = A.e4m3_rows(x)
    assert list(byte.astype(int) - 127) == [120, 120, 119]
    got = A.e4m3_values(codes, byte)
    assert np.array_equal(got[0], [240 * 2.0 ** 120, -240 * 2.0 ** 120, 0.0])
    assert np.array_equal(got[1, :2], [240 * 2.0 ** 120] * 2) and np.isnan(got[1, 2])
    assert np.array_equal(got[2], [2.0 ** 127, 224 * 2.0 ** 119, 0.0])


@pytest.mark.parametrize("per,heads,io", [(1, 1, 1), (1, 2, 1), (1, 8, 1), (16, 1, 1), (30, 2, 1), (200, 4, 1), (40, 1, 0)])
def test_launches_at_their_limit(per, heads, io):
    """The header's formula at 2^24 workgroups, for `per` tokens a request of ungrouped heads: tiles of 16 rows
    up to 16 tokens, of 32 for fp32, else of 128."""
    a = lkv.Attn(h_q=heads, h_kv=heads, d=128, page=64, io_dtype=io, cache_dtype=io, scale=0.1)
    rows = 32 if io == 0 else 16 if per <= 16 else 128

    def status(r):
        return lkv.load().lkv_attn_paged_workspace(a, r, r * per, 1, ctypes.byref(ctypes.c_size_t(0)))

    lo, hi = 1, 1 << 24  # lo requests are fewer than 2^24 workgroups, hi are not
    while hi - lo > 1:
        r = (lo + hi) // 2
        lo, hi = (r, hi) if (r + (r * per - 1) // rows) * heads < 1 << 24 else (lo, r)
    assert status(lo) == 0 and status(hi) == 2 and hi * per * heads < 1 << 31
