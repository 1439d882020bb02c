"""Oracle of the 8-bit matrices: E4M3 codes (OCP 8-bit floating point specification) with a binary32 scale for each block
of 128 elements of a row, or of 128 x 128, and the product of two such matrices.

TEST INFRASTRUCTURE ONLY: plain numpy; the product path (the HIP library) shares no code with it.  The scale is
max(amax / 448, 2^-126), amax over the finite magnitudes of the block, and the code is that of x * (1 / scale); quotient,
reciprocal and product are binary32 operations (numpy's), the code is found in the table of all values: the nearest one,
ties to the even code, magnitudes over 448 to 448, NaN to NaN.
"""
import numpy as np

BLOCK = 128


def _table():
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        mag = np.ldexp(f / 8.0, -6) if e == 0 else np.ldexp(1 + f / 8.0, e - 7)
        v[c] = np.nan if (c & 127) == 127 else (-mag if c & 128 else mag)
    return v


VALUES = _table()
POSITIVE = VALUES[:127]


def encode(y):
    """E4M3 codes of binary32 numbers."""
    y = np.asarray(y, dtype=np.float32).astype(np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(y), 0.0, y)), 448.0)
    hi = np.searchsorted(POSITIVE, a)                      # first value >= a
    lo = np.maximum(hi - 1, 0)
    down, up = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(y), 127, code)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantize(x, blocks="rows"):
    """(codes, scales): scales [ceil(cols/128)][rows] for rows, [ceil(rows/128)][ceil(cols/128)] for tiles."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    cb, rb = -(-cols // BLOCK), -(-rows // BLOCK)
    codes = np.empty((rows, cols), np.uint8)
    scales = np.empty((cb, rows) if blocks == "rows" else (rb, cb), np.float32)
    mag = np.where(np.isfinite(x), np.abs(x), np.float32(0))
    with np.errstate(all="ignore"):
        for c in range(cb):
            cs = slice(c * BLOCK, (c + 1) * BLOCK)
            if blocks == "rows":
                s = np.maximum(mag[:, cs].max(1) / np.float32(448), np.float32(2.0 ** -126))
                scales[c] = s
                codes[:, cs] = encode(x[:, cs] * (np.float32(1) / s)[:, None])
            else:
                for r in range(rb):
                    rs = slice(r * BLOCK, (r + 1) * BLOCK)
                    s = np.maximum(mag[rs, cs].max() / np.float32(448), np.float32(2.0 ** -126))
                    scales[r, c] = s
                    codes[rs, cs] = encode(x[rs, cs] * (np.float32(1) / s))
    return codes, scales


def values(codes, scales, blocks="rows"):
    """What the matrix stands for, in 64 bits."""
    rows, cols = codes.shape
    c = np.arange(cols) // BLOCK
    s = scales.astype(np.float64)
    per = s[c].T if blocks == "rows" else s[np.arange(rows) // BLOCK][:, c]
    return VALUES[codes] * per


def matmul(a, sa, b, sb, b_blocks="tiles", bias=None):
    """(a b^T + bias, the same sum over magnitudes) in 64 bits."""
    va, vb = values(a, sa), values(b, sb, b_blocks)
    y, mag = va @ vb.T, np.abs(va) @ np.abs(vb).T
    return (y, mag) if bias is None else (y + bias, mag + np.abs(bias))
