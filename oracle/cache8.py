"""Tokens into the paged cache in 64 bits: rotary positions, and the 8-bit form (e4m3 numbers, a power of two for each block of 16
tokens and KV head).  Written from the definitions; numpy on whole sequences, one at a time.  (The rotation is the published one of
the architecture the paper names; the paper has no 8-bit cache.)"""
import numpy as np

BLOCK = 16
LEAST = -100

# every finite e4m3 number: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are NaN
_CODE = np.arange(256)
_EXP, _MAN = _CODE >> 3 & 15, _CODE & 7
VALUE = np.where(_EXP == 0, _MAN * 2.0 ** -9, (8 + _MAN) * 2.0 ** (_EXP - 10.0)) * np.where(_CODE & 128, -1.0, 1.0)
VALUE[[0x7f, 0xff]] = np.nan
_UP = VALUE[:127]                                     # non-negative, ascending: the code is the place


def round_e4m3(x):
    """Codes of the nearest numbers, ties to the even code; NaN for what is not finite.  |x| <= 448."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert (a <= 448).all()
    hi = np.searchsorted(_UP, a)                      # first number >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _UP[hi] - a, a - _UP[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == _UP[hi], hi, code)
    return np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 0x7f).astype(np.uint8)


def border_distance(x):
    """How far |x| is from the nearest place where round_e4m3 changes."""
    a = np.abs(np.asarray(x, np.float64))
    ties = (_UP[1:] + _UP[:-1]) / 2
    i = np.searchsorted(ties, a)
    return np.minimum(np.abs(a - ties[np.maximum(i - 1, 0)]), np.abs(ties[np.minimum(i, len(ties) - 1)] - a))


def exponent(amax):
    """Smallest e >= LEAST with amax <= 448 * 2^e."""
    amax = np.asarray(amax, np.float64)
    e = np.full(amax.shape, LEAST, np.int64)
    some = amax > 0
    e[some] = np.maximum(LEAST, np.ceil(np.log2(amax[some]) - np.log2(448.0)).astype(np.int64) - 1)
    while True:                                       # (the logarithm is only where to begin)
        low = amax > np.ldexp(448.0, e)
        if not low.any():
            return e
        e[low] += 1


def rotate(x, pos, theta):
    """x [n, H, dh] at positions pos [n]: pairs (x[2i], x[2i+1]) turned by pos * theta^(-2i/dh)."""
    if theta == 0:
        return np.asarray(x, np.float64)
    dh = x.shape[-1]
    angle = np.asarray(pos, np.float64)[:, None, None] * theta ** (-2.0 * np.arange(dh // 2) / dh)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * angle)
    out = np.empty(x.shape)
    out[..., 0::2], out[..., 1::2] = z.real, z.imag
    return out


def append8(codes, scale, table, length, x):
    """n new rows x [n, Hkv, dh] (float64, rotated) of ONE sequence whose length becomes `length`, into codes [n_pages, Hkv, page, dh]
    and scale [n_pages, Hkv, page / 16] (uint8, in place).  Returns [(page, block in page, first new row, end, exponents)]."""
    n, page, start, done = len(x), codes.shape[2], length - len(x), []
    if n == 0:
        return done
    for lo in range(start // BLOCK * BLOCK, length, BLOCK):
        p, i = table[lo // page], lo % page // BLOCK
        a, b = max(start - lo, 0), min(length - lo, BLOCK)
        rows = x[lo + a - start:lo + b - start]       # [rows, Hkv, dh]
        finite = np.where(np.isfinite(rows), np.abs(rows), 0.0)
        e = exponent(finite.max((0, 2)))
        old = codes[p, :, i * BLOCK:i * BLOCK + a]
        if a:
            was = scale[p, :, i].astype(np.int64) - 127
            e = np.maximum(e, was)
            grown = e > was
            old[grown] = round_e4m3(VALUE[old[grown]] * np.exp2(was - e)[grown, None, None])
        codes[p, :, i * BLOCK + a:i * BLOCK + b] = round_e4m3(rows * np.exp2(-e)[None, :, None]).transpose(1, 0, 2)
        scale[p, :, i] = e + 127
        done.append((p, i, a, b, e))
    return done
