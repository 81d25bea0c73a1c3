"""Microscaled (MX) tensors and the layer on them, written out from their definition (OCP Microscaling Formats 1.0).

TEST INFRASTRUCTURE ONLY.  A block is 32 consecutive elements of a row.  Readings:

  rotation   v = H_32 x / sqrt(32): binary32, strides 16, 8, 4, 2, 1, (a, b) -> (a + b, a - b), then one product with the
             binary32 number nearest to 1/sqrt(32) (rounding decisions depend on it, so the order is fixed)
  scale      2^e, e = floor(log2 max|v|) - emax, emax the exponent of the element type's largest number, e in
             [-127, 127]; a block of zeros: -127; a block with an infinity or a NaN: the scale is NaN (byte 255), codes 0
  element    the representable number nearest to v / 2^e by exhaustive search, ties to the even code, saturating
  products   exact, in binary64

Pins: tests/test_oracle_mx.py.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# E4M3: bias 7, no infinities, code 127 is NaN: the 127 magnitudes below it
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
GRID = {4: E2M1, 8: E4M3}
EMAX = {4: 2, 8: 8}


def rotate(x: np.ndarray, g: int) -> np.ndarray:
    """Rows of binary32 x, blocks of g in (1, 32)."""
    v = np.asarray(x, np.float32)
    if g == 1:
        return v
    shape, h = v.shape, 16
    with np.errstate(all="ignore"):
        while h:
            b = v.reshape(-1, 2, h)
            v = np.stack((b[:, 0] + b[:, 1], b[:, 0] - b[:, 1]), axis=1)
            h //= 2
        return v.reshape(shape) * np.float32(1 / np.sqrt(32.0))


def quantize(x: np.ndarray, bits: int, g: int = 1):
    """binary32 rows -> (codes [rows, cols] with the sign in the top bit of `bits`, scale bytes [rows, cols / 32])."""
    v = rotate(x, g)
    rows, cols = v.shape
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, cols // BLOCK), np.uint8)
    grid = GRID[bits]
    even = np.arange(len(grid)) % 2 * 1e-9                     # of two grid points equally far, the even code
    for r in range(rows):
        for b in range(cols // BLOCK):
            w = v[r, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
            if not np.isfinite(w).all():
                scales[r, b] = 255
                continue
            top = np.abs(w).max()
            e = -127 if top == 0 else int(np.clip(int(np.frexp(top)[1]) - 1 - EMAX[bits], -127, 127))
            scales[r, b] = e + 127
            t = w * 2.0 ** -e
            # distances are exact here (few bits each), so a tie is an exact tie
            far = np.abs(np.abs(t)[:, None] - grid[None, :])
            codes[r, b * BLOCK:(b + 1) * BLOCK] = np.argmin(far + even * grid.max() * 1e-6 * (far == far.min(1, keepdims=True)), axis=1) | (
                np.signbit(t).astype(np.uint8) << (bits - 1))
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray, bits: int) -> np.ndarray:
    """binary64 values of codes and scale bytes."""
    top = 1 << (bits - 1)
    mag = np.append(GRID[bits], np.nan)[codes & (top - 1)] if bits == 8 else GRID[bits][codes & (top - 1)]
    v = np.where(codes & top, -mag, mag)
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(scale, BLOCK, axis=1)


def pack(codes: np.ndarray, bits: int) -> np.ndarray:
    """Bytes as the library stores them: E2M1 codes two to a byte, element 0 in the low nibble."""
    return codes if bits == 8 else (codes[:, 0::2] | codes[:, 1::2] << 4)


def unpack(packed: np.ndarray, bits: int) -> np.ndarray:
    return packed if bits == 8 else np.stack((packed & 15, packed >> 4), axis=2).reshape(packed.shape[0], -1)


def tile(scales: np.ndarray) -> np.ndarray:
    """Scale bytes [rows, blocks] in the library's order, one byte after the other."""
    rows, blocks = scales.shape
    bands, groups = -(-rows // 128), -(-blocks // 4)
    out = np.zeros(bands * groups * 512, np.uint8)
    for r in range(rows):
        for b in range(blocks):
            out[((r // 128) * groups + b // 4) * 512 + 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4] = scales[r, b]
    return out


def hadamard(g: int) -> np.ndarray:
    i = np.arange(g)
    return np.where([[bin(a & b).count("1") % 2 for b in i] for a in i], -1.0, 1.0) / np.sqrt(g)


def inverse(d: np.ndarray, g: int) -> np.ndarray:
    """The inverse of the orthonormal block rotation (its own transpose), binary64."""
    return d if g == 1 else (d.reshape(-1, g) @ hadamard(g)).reshape(d.shape)


def backward(dy: np.ndarray, xv: np.ndarray, wv: np.ndarray, g: int):
    """dx, dw of y = x w^T straight through the rounding, and the sums of magnitudes that bound their errors."""
    dy = dy.astype(np.float64)
    spread = lambda t: t if g == 1 else np.repeat(t.reshape(t.shape[0], -1, g).sum(2) / np.sqrt(g), g, axis=1)  # noqa: E731
    return (inverse(dy @ wv, g), inverse(dy.T @ xv, g), spread(np.abs(dy) @ np.abs(wv)), spread(np.abs(dy).T @ np.abs(xv)))
