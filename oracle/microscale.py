"""Plain definition of the microscaled 4-bit format (numpy, 64 bits): quantizer, values, inner product.

A block of 16 or 32 elements of a row shares a scale; an element is the nearest E2M1 number to x / step, ties to
the number of even place, with the sign of x.  Shares nothing with the CUDA path.
"""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# E4M3 without sign: exponent field e, mantissa m; the largest is 448 (field 15, mantissa 6)
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])[:127]
FLT_MAX = float(np.finfo(np.float32).max)


def nearest(v, numbers):
    """Place of the nearest of the ascending `numbers` to each v >= 0; halfway, the even place; beyond the last, the last."""
    mids = (numbers[1:] + numbers[:-1]) / 2
    below, upto = np.searchsorted(mids, v, side="left"), np.searchsorted(mids, v, side="right")
    return np.where(below % 2 == 0, below, upto)


def quantize(x, block, exp=0, relu=False):
    """x [rows][inner] -> (codes uint8 [rows][inner], scale bytes uint8 [rows][blocks], (zeros, sat_pos, sat_neg))."""
    x = np.asarray(x, dtype=np.float64)
    rows, inner = x.shape
    x = np.clip(np.where(np.isnan(x), 0.0, x), -FLT_MAX, FLT_MAX)
    if relu:
        x = np.where(x > 0, x, 0.0)
    blocks = -(-inner // block)
    full = np.zeros((rows, blocks * block))
    full[:, :inner] = x
    full = full.reshape(rows, blocks, block)
    top = np.abs(full).max(axis=2)
    if block == 32:
        _, e = np.frexp(top)                     # top = f 2^e, 0.5 <= f < 1: floor(log2 top) = e - 1
        byte = np.where(top > 0, np.clip(e - 3, -127, 127) + 127, 0)
        step = np.ldexp(1.0, byte - 127)
    else:
        byte = nearest(np.ldexp(top, -exp) / 6, E4M3)
        step = np.ldexp(E4M3[byte], exp)
    at = step[:, :, None]
    ratio = np.abs(full) / np.where(at > 0, at, np.inf)
    code = nearest(ratio, E2M1) | np.where(np.signbit(full), 8, 0)
    flat = lambda a: a.reshape(rows, -1)[:, :inner]  # noqa: E731
    code, clipped, neg = flat(code).astype(np.uint8), flat(ratio >= 7), flat(np.signbit(full))
    counts = (int(((code & 7) == 0).sum()), int((clipped & ~neg).sum()), int((clipped & neg).sum()))
    return code, byte.astype(np.uint8), counts


def values(code, byte, block, exp=0):
    """What the codes stand for, in 64 bits (exact)."""
    code, byte = np.asarray(code), np.asarray(byte).astype(np.int64)
    if block == 32:
        step = np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))
    else:
        step = np.where(byte == 127, np.nan, np.ldexp(E4M3[np.minimum(byte, 126)], exp))
    v = E2M1[code & 7] * np.repeat(step, block, axis=1)[:, :code.shape[1]]
    return np.where(code & 8, -v, v)


def inner_product(x, w, bias=None, relu=False):
    y = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return np.maximum(y, 0.0) if relu else y


# ---- storage
def pack_codes(code, c_stride):
    rows, inner = code.shape
    full = np.zeros((rows, c_stride), np.uint8)
    full[:, :inner] = code
    return full[:, 0::2] | (full[:, 1::2] << 4)


def unpack_codes(data, inner):
    full = np.stack([data & 15, data >> 4], axis=2).reshape(data.shape[0], -1)
    return full[:, :inner]


def scale_places(rows, inner, block):
    """Offset in the scale plane of every row's blocks, and of the bytes that fill the row's last tile up."""
    blocks = -(-inner // block)
    groups = -(-blocks // 4)
    r, j = np.arange(rows)[:, None], np.arange(groups * 4)[None, :]
    at = (r // 128 * groups + j // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4
    return at[:, :blocks], at[:, blocks:]
