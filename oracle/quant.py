"""The quantised paged cache in float64, from its definition (include/gvc.h):
a head as e4m3 codes and one e8m0 scale, and what they stand for.

Attention over it is oracle/paged.py's over these values.
"""
import numpy as np

# what the 256 e4m3 codes stand for: sign, 4 exponent bits of bias 7, 3 fraction bits
_c = np.arange(128)
_half = np.where(_c < 8, _c * 2.0 ** -9, (1 + _c % 8 / 8) * 2.0 ** (_c // 8 - 7.0))
_half[127] = np.nan
E4M3 = np.concatenate([_half, -_half])

# the largest code of the 16-bit type that a value past it becomes
MOST = {"bf16": 1.875 * 2.0 ** 127, "fp16": 61440.0}


def scale_code(x):
    """e8m0 code of a head x: the least e >= -126 with max |x| <= 448 * 2^e, as e + 127 (finite values count)."""
    size = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = -126
    while size > 448 * 2.0 ** e:
        e += 1
    return e + 127


def bounded(x, t):
    return np.where(np.isfinite(x), np.clip(x, -MOST[t], MOST[t]), x)


def quantise(x, t):
    """(codes uint8, scale code) of a head vector x."""
    x = bounded(np.asarray(x, dtype=np.float64), t)
    code = scale_code(x)
    return _nearest(x, code - 127), code


def _nearest(x, e):
    """Codes nearest to x / 2^e, the even one of two."""
    y = np.abs(x) / 2.0 ** np.asarray(e, dtype=np.float64)
    i = np.clip(np.searchsorted(_half[:127], y, side="right") - 1, 0, 125)   # _half[i] <= y
    low, high = y - _half[i], _half[i + 1] - y
    c = np.where((high < low) | ((high == low) & (i % 2 == 1)), i + 1, i)
    c = np.where(np.isfinite(x), c, 127)
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def quantise_heads(x, t):
    """quantise() of all heads of x [..., dh] at once."""
    x = bounded(np.asarray(x, dtype=np.float64), t)
    size = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    e = np.frexp(size / 448)[1]
    e = np.where(448 * 2.0 ** (e - 1.0) >= size, e - 1, e)   # a power of two is its own bound
    e = np.where(size > 0, np.maximum(e, -126), -126)
    return _nearest(x, e[..., None]), (e + 127).astype(np.uint8)


def values(codes, scales, t):
    """What codes [..., dh] with scale codes [...] stand for, rounded to the 16-bit type."""
    x = E4M3[codes] * np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))[..., None]
    with np.errstate(over="ignore"):
        if t == "fp16":
            return x.astype(np.float16).astype(np.float64)
        # bf16: eight bits of fraction hold a code's four, down to the step 2^-133 and up to 2^128
        x = np.where(np.abs(x) < 2.0 ** -126, np.round(x * 2.0 ** 133) * 2.0 ** -133, x)
        return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)
