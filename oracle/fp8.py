"""TEST INFRASTRUCTURE: 8-bit floating point with a scale for each block of 128, and the product of such operands.

e4m3: a sign, 4 exponent bits with bias 7, 3 mantissa bits; exponent 0 holds i * 2^-9, exponent e the values (1 + i/8) * 2^(e-7); the
code 0x7f (and 0xff) is a NaN, so the largest value is 1.75 * 2^8 = 448.  The quantizer is evaluated in float32, one
rounding per operation, since a code is a whole number decided by floating point; the product is evaluated in float64.
Nothing here is shared with the HIP path.
"""
from __future__ import annotations

import numpy as np

F = np.float32
BLOCK = 128


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    out = np.empty(256)
    for c in range(256):
        e, i = (c >> 3) & 15, c & 7
        v = i * 2.0 ** -9 if e == 0 else (1 + i / 8) * 2.0 ** (e - 7)
        if e == 15 and i == 7:
            v = np.nan
        out[c] = -v if c & 128 else v
    return out


_TABLE = e4m3_values()
_POSITIVE = _TABLE[:127]                      # rising, 0 .. 448


def e4m3_codes(v) -> np.ndarray:
    """The codes nearest to v (|v| <= 448 and a little), ties to the even code, the sign kept."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(np.isnan(v), np.uint8(127), code)
    return code | np.where(np.signbit(v) & ~np.isnan(v), np.uint8(128), np.uint8(0))


def quantize_fp8(x, block_rows: int):
    """(codes [rows, cols] uint8, scales) of a float32 matrix, a scale for each block of block_rows x 128."""
    x = np.asarray(x, F)
    rows, cols = x.shape
    nr, nb = -(-rows // block_rows), -(-cols // BLOCK)
    codes, scales = np.empty((rows, cols), np.uint8), np.empty((nr, nb), F)
    for i in range(nr):
        for j in range(nb):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            top = np.abs(x[at]).max()
            if not np.isfinite(top):
                codes[at], scales[i, j] = 127, np.nan
                continue
            s = F(top / F(448))
            if s < F(2.0 ** -126):
                s = F(1)
            inv = F(F(1) / s)
            codes[at], scales[i, j] = e4m3_codes((x[at] * inv).astype(F)), s
    return codes, scales


def dequantize_fp8(codes, scales, block_rows: int) -> np.ndarray:
    """float64 values of the codes."""
    rows, cols = codes.shape
    s = np.repeat(np.repeat(np.asarray(scales, np.float64), block_rows, 0)[:rows], BLOCK, 1)[:, :cols]
    return _TABLE[codes] * s


def ref_fp8_matmul(x, x_scales, w, w_scales):
    """(y, the sum of the products' magnitudes) in float64: y = x w^T."""
    a, b = dequantize_fp8(x, x_scales, 1), dequantize_fp8(w, w_scales, BLOCK)
    return a @ b.T, np.abs(a) @ np.abs(b).T
