"""fp64 oracle: microscaled 4-bit floating point (MXFP4).

TEST INFRASTRUCTURE ONLY (see the package docstring).

A row is cut into blocks of 32 elements; a block has one scale byte s and 32
codes of 4 bits (sign, two bits of exponent x, one of mantissa m):

    value = (-1)^sign * M * 2^(s - 127),
    M = m / 2 for x = 0, (1 + m / 2) * 2^(x - 1) otherwise;  s = 255: NaN.

Two codes share a byte, the element of lower index in the low nibble.
Quantising: with top the largest magnitude of the block, s - 127 is
floor(log2 top) - 2, at least -127 (and -127 for a block of zeros); codes are the
nearest of the eight magnitudes, ties to the even code, at most 6.  A block with
a value that is not finite has s = 255 and codes 0.
"""
import numpy as np

MAGNITUDES = np.array([m / 2 if x == 0 else (1 + m / 2) * 2.0 ** (x - 1)
                       for x in range(4) for m in range(2)])


def values(codes, scales):
    """codes [..., n/2], scales [..., n/32] (uint8) -> values [..., n] in fp64."""
    c = np.asarray(codes)
    nib = np.stack([c & 15, c >> 4], axis=-1).reshape(c.shape[:-1] + (2 * c.shape[-1],))
    v = MAGNITUDES[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    e = np.repeat(np.asarray(scales).astype(np.int64) - 127, 32, axis=-1)
    out = v * 2.0 ** e.astype(np.float64)
    return np.where(e == 128, np.nan, out)


def quantize(x):
    """x [..., n] (values exact in fp64) -> (codes [..., n/2], scales [..., n/32]) uint8."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(-1, 32)
    finite = np.isfinite(b).all(axis=1)
    a = np.abs(np.where(finite[:, None], b, 0.0))
    top = a.max(axis=1)
    # frexp: top = f 2^k with f in [0.5, 1), so floor(log2 top) = k - 1
    e = np.where(top > 0, np.maximum(np.frexp(top)[1] - 3, -127), -127)
    r = np.ldexp(a, -e[:, None])
    d = np.abs(r[:, :, None] - MAGNITUDES)
    near = d == d.min(axis=2, keepdims=True)
    # of two nearest codes (a tie) the even one
    first, last = near.argmax(axis=2), 7 - near[:, :, ::-1].argmax(axis=2)
    code = np.where(first == last, first, np.where(first % 2 == 0, first, last))
    code = code + 8 * (np.signbit(b) & finite[:, None])
    codes = (code[:, 0::2] + 16 * code[:, 1::2]).astype(np.uint8)
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    n = x.shape[-1]
    return codes.reshape(x.shape[:-1] + (n // 2,)), scales.reshape(x.shape[:-1] + (n // 32,))


def rounded(x):
    """The values that x is held as."""
    return values(*quantize(x))
