"""A cache of 8 bits, plain: e4m3 by its fields, the exponent of a block, and the
rows of one block of one head as an append leaves them.  fp64."""

import numpy as np

RANGE = {"fp16": (-15, 8), "bf16": (-117, 120)}     # exponents of a block
MOST = {"fp16": 1.875 * 2.0 ** 15, "bf16": 1.875 * 2.0 ** 127}


def decode(codes):
    """e4m3: (1 + f / 8) 2^(x - 7), f / 8 2^-6 for x = 0, NaN for x = 15 and f = 7."""
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    x, f = (c >> 3) & 15, c & 7
    size = np.where(x > 0, (8 + f) * 2.0 ** (x - 10), f * 2.0 ** -9)
    size = np.where((x == 15) & (f == 7), np.nan, size)
    return np.where(c >= 128, -size, size)


_VALUES = decode(np.arange(127))                     # ascending, 0 .. 448


def encode(x):
    """The nearest code, ties to the even one; |x| <= 464; NaN to 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.nan_to_num(x, nan=0.0))
    assert (a <= 464).all()
    hi = np.searchsorted(_VALUES, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _VALUES[hi] - a, a - _VALUES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def exponent(most, dtype):
    lo, hi = RANGE[dtype]
    e = lo
    while e < hi and most > 448 * 2.0 ** e:
        e += 1
    return e


def append(old, e_old, new, dtype):
    """old [rows before][D] codes under 2^e_old, new [rows][D] values -> (codes of all of them, exponent)."""
    new = np.asarray(new, dtype=np.float64)
    fine = np.isfinite(new)
    x = np.where(fine, np.clip(np.where(fine, new, 0), -MOST[dtype], MOST[dtype]), np.nan)
    e = exponent(np.abs(np.where(fine, x, 0)).max(initial=0), dtype)
    kept = np.asarray(old, dtype=np.uint8)
    if len(kept):
        e0 = min(max(e_old, RANGE[dtype][0]), RANGE[dtype][1])
        if e0 >= e:
            e = e0
        else:
            kept = encode(decode(kept) * 2.0 ** (e0 - e)) | (kept & 128)
    return np.concatenate([kept.reshape(-1, new.shape[1]), encode(x / 2.0 ** e)]), e
