"""TEST INFRASTRUCTURE ONLY -- the 8-bit KV cache by definition, in 64 bits with numpy.

A cache here is a dict of numpy arrays: "k", "v" uint8 e4m3 bytes [rows, Hkv, d], "k_scale", "v_scale" uint8 exponent bytes
[blocks, Hkv], "block".  A row's value is its byte's value times 2^(scale byte - 127).
"""

from __future__ import annotations

import numpy as np

SCALE_MIN, SCALE_MAX = 10, 246


def _table():
    """The 256 values of e4m3: sign, four bits of exponent (bias 7), three of fraction; all ones is NaN, no infinities."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * np.exp2(e - 10.0))
    x[(b & 127) == 127] = np.nan
    return np.where(b & 128, -x, x)


E4M3 = _table()


def encode(x):
    """Nearest e4m3 bytes of float64 values within [-448, 448], ties to the even byte; zeros keep their sign."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    grid = E4M3[:127]
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_byte(top):
    """The smallest power of two (as its byte) that brings a magnitude to 448 or below, within the bytes allowed."""
    for e in range(SCALE_MIN, SCALE_MAX):
        if top <= 448.0 * 2.0 ** (e - 127):
            return e
    return SCALE_MAX


def values(cache, which, rows=None):
    x, s = cache[which], cache[which + "_scale"]
    rows = np.arange(x.shape[0]) if rows is None else np.asarray(rows)
    return E4M3[x[rows]] * np.exp2(s[rows // cache["block"]].astype(np.float64) - 127.0)[..., None]


def store(cache, rows, k, v):
    """Token i (k[i], v[i]: float64 [Hkv, d]) into row rows[i], block by block and head by head; in place."""
    rows, B = np.asarray(rows), cache["block"]
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))  # [n, Hkv]
    for b in np.unique(rows // B):
        mine = np.nonzero(rows // B == b)[0]
        low = int((rows[mine] % B).min())
        kept = np.arange(b * B, b * B + low)
        for which, x in (("k", k), ("v", v)):
            for h in range(x.shape[1]):
                good = mine[~bad[mine, h]]
                top = np.abs(x[good, h]).max() if good.size else 0.0
                e, old = scale_byte(top), int(cache[which + "_scale"][b, h])
                if low > 0:
                    e = max(e, old)
                    if e > old:
                        y = E4M3[cache[which][kept, h]]
                        nan = np.isnan(y)
                        cache[which][kept, h] = np.where(nan, cache[which][kept, h], encode(np.where(nan, 0, y) * 2.0 ** (old - e)))
                cache[which + "_scale"][b, h] = e
                for i in mine:
                    if bad[i, h]:
                        cache[which][rows[i], h] = 127 if which == "k" else 0
                    else:
                        cache[which][rows[i], h] = encode(x[i, h] * 2.0 ** (127 - e))
