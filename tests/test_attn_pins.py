"""Pins of the attention oracle: closed forms, and the e4m3 format against torch's."""
import numpy as np
import torch

from oracle import attention as A


def test_equal_keys_give_the_mean():
    v = np.arange(12.0).reshape(6, 1, 2)
    o, mag, _ = A.attention(np.ones((3, 2, 2)), np.ones((6, 1, 2)), v, [0, 2, 5], 0.7)
    for i, m in enumerate((1, 3, 6)):
        assert np.allclose(o[i], v[:m, 0].mean(axis=0)) and np.allclose(mag[i], o[i])


def test_two_keys_by_hand():
    # scores 0 and ln 3: weights 1/4 and 3/4
    o, _, dot = A.attention([[[1.0]]], [[[0.0]], [[np.log(3.0)]]], [[[8.0]], [[-4.0]]], [1], 1.0)
    assert np.allclose(o, 8 / 4 - 3.0) and np.allclose(dot, np.log(3.0))


def test_heads_share_keys_and_empty_rows_are_zero():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((2, 4, 3)), rng.standard_normal((5, 2, 3)), rng.standard_normal((5, 2, 3))
    o, _, _ = A.attention(q, k, v, [4, -1], 1.0)
    assert not o[1].any()
    for h in range(4):
        one, _, _ = A.attention(q[:1, h:h + 1], k[:, h // 2:h // 2 + 1], v[:, h // 2:h // 2 + 1], [4], 1.0)
        assert np.allclose(o[0, h], one[0, 0])


def test_e4m3_against_torch():
    codes = np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(A.e4m3_values(codes[None], np.array([127]))[0], t)
    rng = np.random.default_rng(1)
    mid = (A.E4M3[:-1] + A.E4M3[1:]) / 2  # ties
    y = np.concatenate([rng.uniform(-448, 448, 3000), rng.uniform(-0.05, 0.05, 3000), mid, -mid, A.E4M3, [np.nan]])
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = A.e4m3_codes(y.astype(np.float32))
    assert np.array_equal(got[:-1], want[:-1]) and got[-1] & 0x7f == want[-1] & 0x7f == 0x7f


def test_row_scale():
    x = np.array([[448.0, 1.0], [448.5, 0.0], [0.0, 0.0], [np.inf, 1.75], [2.0 ** 127, 0.0], [2.0 ** -130, 0.0]])
    _, b = A.e4m3_rows(x)
    assert list(b.astype(int) - 127) == [0, 1, -100, -8, 119, -100]
