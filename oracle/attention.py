"""Causal attention and the e4m3 cache format in fp64, straight from their definitions."""
import numpy as np


def attention(q, k, v, pos, scale):
    """o[i, h] = sum_j p_ij v[j, h'] over the keys j <= pos[i], h' = h / (h_q / h_kv), with p_ij
    the softmax of scale * q.k; zeros where no key is seen.  q [n, h_q, d], k, v [c, h_kv, d].
    Also returns sum_j p_ij |v[j]|, the scale of the result's rounding errors, and the largest
    sum_e |q_e k_e| * scale of each row."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, hq, d = q.shape
    hkv = k.shape[1]
    o, mag, dot = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq))
    for i in range(n):
        m = min(int(pos[i]) + 1, k.shape[0])
        if m <= 0:
            continue
        for h in range(hkv):
            g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            s = scale * (q[i, g] @ k[:m, h].T)
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            o[i, g] = p @ v[:m, h]
            mag[i, g] = p @ np.abs(v[:m, h])
            dot[i, g] = scale * (np.abs(q[i, g]) @ np.abs(k[:m, h]).T).max(axis=1)
    return o, mag, dot


# every non-negative e4m3 value by its code: subnormals m 2^-9, then (8 + m) 2^(e - 10); 0x7f is NaN
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(0x7f)])


def e4m3_codes(y):
    """Nearest e4m3 codes of |y| <= 448, ties to the even code; NaN for what is not finite."""
    y = np.asarray(y, np.float64)
    a = np.abs(np.where(np.isfinite(y), y, 0.0))
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.isfinite(y), c, 0x7f)
    return (c | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def e4m3_rows(x):
    """Codes and exponent bytes of rows x [..., d].  At the largest scale magnitudes stop at 240 * 2^120, the
    largest that bf16 holds too."""
    x = np.asarray(x, np.float64)
    amax = np.max(np.abs(np.where(np.isfinite(x), x, 0.0)), axis=-1)
    e = np.full(amax.shape, -100)
    for i in np.ndindex(amax.shape):
        while e[i] < 120 and amax[i] > 448.0 * 2.0 ** e[i]:
            e[i] += 1
    y = x * 2.0 ** -e[..., None].astype(np.float64)
    y = np.where((e[..., None] == 120) & np.isfinite(y), np.clip(y, -240.0, 240.0), y)
    return e4m3_codes(y), (e + 127).astype(np.uint8)


def e4m3_values(codes, exps):
    codes = np.asarray(codes)
    a = np.append(E4M3, np.nan)[codes & 0x7f]
    return np.where(codes & 0x80, -a, a) * 2.0 ** (np.asarray(exps, np.float64)[..., None] - 127)
