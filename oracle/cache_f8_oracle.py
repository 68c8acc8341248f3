"""Plain 64-bit implementation of the cache in 8-bit numbers (vla_cache.h), from the numbers' definition: sign, 4 bits of
exponent, 3 of mantissa, bias 7, all ones NaN."""
import numpy as np

from .cache_oracle import PAGE

LEAST = 2.0 ** -100


def numbers():
    """The value of each byte."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = np.nan if e == 15 and m == 7 else -x if b & 128 else x
    return out


NUMBERS = numbers()


def encode(x):
    """(bytes, scale of each head as fp32) of x [..., head_dim]: the nearest of x 448 / top, ties to even."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1, keepdims=True)
    bad = ~np.isfinite(top)
    top = np.where(bad, 1.0, np.maximum(top, LEAST))
    y = np.where(bad, 0.0, x) * 448.0 / top
    pos = NUMBERS[:127]  # ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = pos[hi] - a, a - pos[lo]
    b = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    b = b + 128 * np.signbit(y)
    b = np.where(bad, 127, b).astype(np.uint8)
    scale = np.where(bad, np.nan, top)[..., 0].astype(np.float32) / np.float32(448)
    return b, scale


def append(kp, vp, ks, vs, slots, k, v):
    """Copies of the pools (bytes and scales) with row r's key and value at slots[r] (rows outside the pool passed over)."""
    kp, vp, ks, vs = kp.copy(), vp.copy(), ks.copy(), vs.copy()
    kb, vb = encode(k), encode(v)
    for r, s in enumerate(slots):
        if 0 <= s < PAGE * len(kp):
            kp[s // PAGE, :, s % PAGE], ks[s // PAGE, :, s % PAGE] = kb[0][r], kb[1][r]
            vp[s // PAGE, :, :, s % PAGE], vs[s // PAGE, :, s % PAGE] = vb[0][r], vb[1][r]
    return kp, vp, ks, vs


def values(kp, vp, ks, vs):
    """The pools' elements."""
    return NUMBERS[kp] * ks.astype(np.float64)[..., None], NUMBERS[vp] * vs.astype(np.float64)[:, :, None]
