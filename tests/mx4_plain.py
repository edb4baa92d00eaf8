"""The 4-bit format in plain numpy (fp64), for the tests of its operators."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2      # between code i and i + 1


def scale_of(top):
    """The scale byte of groups whose largest magnitudes are given."""
    top = np.asarray(top, dtype=np.float64)
    byte = np.full(top.shape, 2)
    for s in range(3, 253):
        byte[top > 7 * 2.0 ** (s - 1 - 127)] = s
    byte[~np.isfinite(top)] = 255
    return byte


def codes_of(x, byte):
    """The codes of values x with the scale bytes given (the same shape)."""
    y = x * 2.0 ** (127.0 - byte)
    mag = np.abs(y)
    code = np.zeros(x.shape, dtype=np.int64)
    for i, border in enumerate(BORDERS):      # a tie goes to the even one of i and i + 1
        code += (mag > border) | ((mag == border) & (i % 2 == 1))
    return np.where(byte == 255, 0, code + 8 * np.signbit(y))


def values_of(code, byte):
    """What codes with scale bytes (the same shape) stand for."""
    mag = MAGNITUDES[code & 7] * np.where(code >= 8, -1.0, 1.0)
    return np.where(byte == 255, np.nan, mag * 2.0 ** (byte - 127.0))


def group_bytes(x, axis):
    """Scale bytes of x's groups of 32 along `axis`, one for every value of x."""
    x = np.moveaxis(x, axis, -1)
    out = np.empty(x.shape, dtype=np.int64)
    for lo in range(0, x.shape[-1], 32):
        with np.errstate(invalid="ignore"):
            out[..., lo:lo + 32] = scale_of(np.abs(x[..., lo:lo + 32]).max(-1))[..., None]
    return np.moveaxis(out, -1, axis)


def rounded(x, axis=-1):
    """x in 4 bits, as values."""
    byte = group_bytes(x, axis)
    with np.errstate(invalid="ignore"):
        return values_of(codes_of(x, byte), byte)
