"""The operators on FP8 matrices in 64 bits with numpy, from their definitions; used by the tests only."""
import math

import numpy as np

E4M3, E5M2 = 2, 5
TOP = {E4M3: 448.0, E5M2: 57344.0}


def table(fmt):
    """The values of the 256 bytes."""
    bits, bias = (3, 7) if fmt == E4M3 else (2, 15)
    out = np.zeros(256)
    for byte in range(256):
        e, f = (byte & 127) >> bits, byte & ((1 << bits) - 1)
        v = math.ldexp(f, 1 - bias - bits) if e == 0 else math.ldexp(f + (1 << bits), e - bias - bits)
        if fmt == E4M3 and byte & 127 == 127 or fmt == E5M2 and e == 31 and f:
            v = math.nan
        elif fmt == E5M2 and e == 31:
            v = math.inf
        out[byte] = -v if byte & 128 else v
    return out


def encode(v, fmt):
    """Bytes of the values nearest to v (|v| <= TOP), ties to the even byte; NaN as 0x7F or 0xFF, infinities as documented."""
    t = table(fmt)[:127 if fmt == E4M3 else 124]           # 0 and the finite positive values, ascending
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    hi = np.clip(np.searchsorted(t, a), 1, len(t) - 1)
    lo = hi - 1
    d_lo, d_hi = a - t[lo], t[hi] - a
    byte = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    byte = byte | np.where(np.signbit(v), 128, 0)
    if fmt == E5M2:
        byte = np.where(np.isinf(v), 0x7C | np.where(v < 0, 128, 0), byte)
    return byte.astype(np.uint8)


def scale_exponents(x, fmt, block):
    """e of every block of block x 128."""
    rows, cols = x.shape
    nr, nc = -(-rows // block), -(-cols // 128)
    full = np.zeros((nr * block, nc * 128))
    full[:rows, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = full.reshape(nr, block, nc, 128).max(axis=(1, 3))
    e = np.full(amax.shape, -127)
    for i in np.ndindex(*amax.shape):
        if amax[i] > 0:
            k = math.frexp(amax[i] / TOP[fmt])[1]           # amax / top < 2^k
            e[i] = max(-127, k - 1 if amax[i] <= math.ldexp(TOP[fmt], k - 1) else k)
    return e


def quantize(x, fmt, block):
    """(element bytes, scale bytes, mask of the elements that are NaN) of a float64 matrix."""
    e = scale_exponents(x, fmt, block)
    s = np.repeat(np.repeat(e, block, 0)[: x.shape[0]], 128, 1)[:, : x.shape[1]]
    nan = np.isnan(x) | (np.isinf(x) if fmt == E4M3 else False)
    return encode(np.where(nan, 0.0, np.ldexp(np.where(nan, 0.0, x), -s)), fmt), (e + 127).astype(np.uint8), nan


def values(elems, scales, fmt, block):
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    s = np.repeat(np.repeat(s, block, 0)[: elems.shape[0]], 128, 1)[:, : elems.shape[1]]
    return table(fmt)[elems] * s
