"""Matrices of E4M3 codes with one power-of-two scale per block of 128 columns and 1 or 128 rows, in fp64 NumPy.

Element [r, c] is decode(code[r, c]) * 2^(scale[r // block_rows, c // 128] - 127); the scale byte 255 stands for NaN.
"""
from __future__ import annotations

import numpy as np

from . import sdvg_oracle as O


def of_elements(scale: np.ndarray, rows: int, cols: int, block_rows: int) -> np.ndarray:
    """The factor of every element."""
    s = scale[np.arange(rows) // block_rows][:, np.arange(cols) // 128]
    with np.errstate(over="ignore"):
        return np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))


def values(codes: np.ndarray, scale: np.ndarray, block_rows: int) -> np.ndarray:
    with np.errstate(invalid="ignore"):
        return O.e4m3_decode(codes) * of_elements(scale, *codes.shape, block_rows)


def scale_bytes(x: np.ndarray, block_rows: int) -> np.ndarray:
    """e + 127 with e of each block's largest magnitude, NaN elements left out."""
    rows, cols = x.shape
    a = np.where(np.isnan(x), 0.0, np.abs(x))
    out = np.empty((-(-rows // block_rows), -(-cols // 128)), dtype=np.uint8)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            out[i, j] = 127 + O.e4m3_tile_scale_exponent(a[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128].max())
    return out


def quantise(x: np.ndarray, block_rows: int):
    """(codes, scale bytes); the division by a power of two is exact."""
    s = scale_bytes(x, block_rows)
    with np.errstate(invalid="ignore"):
        return O.e4m3_encode(x / of_elements(s, *x.shape, block_rows)), s


def half_step(v: np.ndarray, scale_of_element: np.ndarray) -> np.ndarray:
    """How far rounding to E4M3 moves a value of magnitude v: 2^-4 of it, or half of the subnormals' step, 2^-9 of the scale."""
    return np.maximum(2.0 ** -4 * v, 2.0 ** -10 * scale_of_element)
