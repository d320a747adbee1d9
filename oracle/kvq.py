"""Quantised KV cache, in float64 from the definition: blocks of 32 consecutive elements of a row share the scale 2^e with
e = floor(log2 a) - emax, one more where a / 2^floor(log2 a) >= 1.75 (a = the block's largest magnitude, emax = 8 for e4m3 and 2
for e2m1, e >= -110), and every element is replaced by the nearest number of the element type times the scale, ties to the
even code.  Blocks that hold an infinity, a NaN or a magnitude of 1.75 * 2^127 or more are NaN."""
import math

import numpy as np

BLOCK = 32
EMAX = {"fp8": 8, "fp4": 2}


def kvq_numbers(fmt):
    """The numbers >= 0 of the element type by code (float64): sign-less e4m3 without its NaN, e2m1."""
    man, low, top = (3, -6, 127) if fmt == "fp8" else (1, 0, 8)
    out = []
    for code in range(top):
        exp, frac = code >> man, code & ((1 << man) - 1)
        out.append(math.ldexp(frac, low - man) if exp == 0 else math.ldexp((1 << man) + frac, low + exp - 1 - man))
    return np.array(out)


def kvq_quantise(x, fmt):
    """x [..., D] -> (codes uint8 [..., D], sign in the top bit of the 4 or 8; scale bytes uint8 [..., D / 32])."""
    with np.errstate(invalid="ignore"):                             # (NaN)
        x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    numbers = kvq_numbers(fmt)
    peak = np.abs(b).max(-1)                                        # (NaN where a number is)
    bad = ~(peak < 1.75 * 2.0 ** 127)
    m, e = np.frexp(np.where(bad, 1.0, peak))                       # peak = m 2^e, m in [0.5, 1)
    e = np.where(peak > 0, np.maximum(e - 1 - EMAX[fmt] + (2 * m >= 1.75), -110), -110)
    y = np.ldexp(np.where(bad[..., None], 0.0, np.abs(b)), -e[..., None].astype(np.int64))
    above = np.clip(np.searchsorted(numbers, y), 1, len(numbers) - 1)      # numbers[above - 1] < y <= numbers[above], if any
    lo, hi = y - numbers[above - 1], numbers[above] - y
    codes = np.where((lo > hi) | ((lo == hi) & (above % 2 == 0)), above, above - 1)
    codes = codes + np.where(np.signbit(b) & ~bad[..., None], 128 if fmt == "fp8" else 8, 0)
    return codes.astype(np.uint8).reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def kvq_values(codes, scales, fmt):
    """The numbers (float64 [..., D]) that codes and scale bytes stand for."""
    numbers = kvq_numbers(fmt)
    sign = 128 if fmt == "fp8" else 8
    codes = np.asarray(codes)
    v = numbers[codes % sign] * np.where(codes >= sign, -1.0, 1.0)
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, np.asarray(scales, dtype=np.int64) - 127))
    return (v.reshape(*v.shape[:-1], -1, BLOCK) * scale[..., None]).reshape(v.shape)
