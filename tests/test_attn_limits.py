"""The full-attention layers' format and sizes at their limits, on the CPU."""
import numpy as np

from oracle import attention as A


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
