"""The full-attention layers' format and sizes at their limits, on the CPU."""
import ctypes
import random

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


BOUND_LAYERS = [(8, 8, 128, 1, 1), (32, 8, 128, 1, 1), (32, 8, 128, 1, 2), (16, 2, 256, 1, 1), (16, 2, 256, 1, 2), (6, 1, 64, 1, 1),
                (64, 1, 64, 1, 2), (3, 3, 64, 0, 0), (8, 2, 128, 0, 0), (1, 1, 64, 1, 1)]


@pytest.mark.parametrize("hq,hkv,d,io,cache", BOUND_LAYERS)
def test_a_workspace_for_every_smaller_call(hq, hkv, d, io, cache):
    """The bound over a batch holds for the batch and for every smaller one: all of few requests and tokens,
    and numbers of either spread over their ranges."""
    a = lkv.Attn(h_q=hq, h_kv=hkv, d=d, page=16, io_dtype=io, cache_dtype=cache, scale=0.1)
    rng = random.Random(hq * d + cache)
    spread = lambda hi: int(round(hi ** rng.random()))  # noqa: E731
    calls = [(r, t, p) for r in range(1, 20) for t in range(1, 40) for p in (17, 4096)]
    calls += [(spread(5000), spread(200000), spread(1 << 17)) for _ in range(20000)]
    need = sorted((t, p, lkv.attn_paged_workspace(a, r, t, p)) for r, t, p in calls)
    for n_tok, width in [(1, 4096), (39, 17), (39, 1 << 17), (300, 1 << 10), (5000, 1 << 17), (200000, 1 << 12), (200000, 1 << 17)]:
        bound = lkv.attn_paged_workspace_bound(a, n_tok, width)
        most = max(n for t, p, n in need if t <= n_tok and p <= width)
        assert most <= bound <= 393216 * (4 * d + 8) and (bound == 0) == (most == 0)
    assert lkv.attn_paged_workspace_bound(a, 0, 1 << 17) == lkv.attn_paged_workspace_bound(a, 100, 16) == 0


def test_bound_arguments():
    f, n = lkv.load().lkv_attn_paged_workspace_bound, ctypes.c_size_t(0)
    a = lkv.Attn(h_q=8, h_kv=2, d=128, page=64, io_dtype=1, cache_dtype=1, scale=0.1)
    bad = lkv.Attn(h_q=8, h_kv=2, d=96, page=64, io_dtype=1, cache_dtype=1, scale=0.1)
    assert f(a, 4, 2, None) == f(None, 4, 2, ctypes.byref(n)) == 1 and f(bad, 4, 2, ctypes.byref(n)) == 5
    assert f(a, -1, 2, ctypes.byref(n)) == f(a, 1 << 31, 2, ctypes.byref(n)) == f(a, 4, -1, ctypes.byref(n)) == 2
    assert f(a, 4, 1 << 26, ctypes.byref(n)) == 2


def test_largest_scale():
    """A scale whose product with log2(e) is past fp32's range would make NaN of scores that are 0."""
    n = ctypes.c_size_t(0)
    for scale, status in ((2.0 ** 127, 0), (3e38, 2), (1e-38, 0), (float("inf"), 2)):
        a = lkv.Attn(h_q=8, h_kv=2, d=128, page=64, io_dtype=1, cache_dtype=1, scale=scale)
        assert lkv.load().lkv_attn_paged_workspace(a, 1, 4, 2, ctypes.byref(n)) == status
