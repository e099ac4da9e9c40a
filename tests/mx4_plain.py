"""Microscaled 4-bit floating point by its definition, in numpy and 64 bits: what the library's kernels are held to.
Shares nothing with them."""
import numpy as np

BOOK = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(cols):
    return -(-cols // 128) * 128


def nearest_codes(u):
    """codes of the entries of BOOK nearest to |u| (ties to the even code, beyond the last to the last) with u's sign"""
    a = np.abs(u)
    distance = np.abs(a[..., None] - BOOK)
    code = distance.argmin(-1)                                  # the lower one of two at the same distance
    upper = np.minimum(code + 1, 7)
    tie = np.take_along_axis(distance, upper[..., None], -1)[..., 0] == np.take_along_axis(distance, code[..., None], -1)[..., 0]
    code = np.where(tie & (code % 2 == 1), upper, code)
    return (code + 8 * np.signbit(u)).astype(np.uint8)


def quantize(x):
    """x (rows x cols) as data (rows x padded/2), scales (padded/128 x rows x 4)"""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    p = padded(cols)
    full = np.zeros((rows, p))
    full[:, :cols] = x
    blocks = full.reshape(rows, p // 32, 32)
    with np.errstate(all="ignore"):
        amax = np.abs(blocks).max(-1, initial=0.0)              # NaN where there is one
        s = np.where(amax > 0, np.floor(np.log2(np.where(amax > 0, amax, 1.0))), 2.0)
        # a logarithm may round across a power of two
        s = np.where((amax > 0) & (np.exp2(np.minimum(s, 1000.0)) > amax), s - 1, s)
        s = np.where((amax > 0) & (np.exp2(np.minimum(s + 1, 1000.0)) <= amax), s + 1, s)
        s = np.clip(s - 2, -127, 127)
        bad = ~np.isfinite(amax)
        s = np.where(bad, 0.0, s)
        code = nearest_codes(np.nan_to_num(blocks, nan=0.0, posinf=0.0, neginf=0.0) * np.exp2(-s)[..., None])
    byte = np.where(bad, 255, s + 127).astype(np.uint8)
    code = code.reshape(rows, p)
    data = code[:, 0::2] | (code[:, 1::2] << 4)
    return data, np.ascontiguousarray(byte.reshape(rows, p // 128, 4).transpose(1, 0, 2))


def values(data, scales, cols):
    """the values of data and scales, rows x cols, 64 bits"""
    data, scales = np.asarray(data), np.asarray(scales)
    rows = data.shape[0]
    code = np.stack([data & 15, data >> 4], -1).reshape(rows, -1)
    v = BOOK[code & 7] * np.where(code & 8, -1.0, 1.0)
    byte = scales.transpose(1, 0, 2).reshape(rows, -1).astype(np.int64)
    scale = np.where(byte == 255, np.nan, np.exp2(byte - 127.0))
    return (v.reshape(rows, -1, 32) * scale[..., None]).reshape(rows, -1)[:, :cols]


def random_matrix(rng, rows, cols):
    """normal, rows and columns of very different size, ties, exact zeros and a block of zeros"""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, 1))) * np.exp2(rng.integers(-3, 4, (1, cols)))
    grid = rng.random((rows, cols)) < 0.3
    x = np.where(grid, np.round(x * 8) / 8, x)
    x[rng.random((rows, cols)) < 0.05] = 0.0
    x[rows // 2, :40] = 0.0
    return x
