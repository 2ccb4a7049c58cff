"""Oracle of the microscaled tensors: 4- or 8-bit elements with one power-of-two scale for 32 values, products on them and the norm in front.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): imported by ``tests/`` alone.

Elements are the paper's sign-and-magnitude codes (Sec. 2.1, Eq. 2; ``oracle/npfmt.py``): E2M1 is (4, 1) at alpha = 1/2, E4M3 is (8, 3) at
alpha = 2^-9 without its last code of each sign, which stands for NaN.  A block of 32 values has its own alpha = 2^(s - 127).  Everything is
computed in 64 bits, where element values, scales and quotients by powers of two are exact.
"""
from __future__ import annotations

import numpy as np

from oracle import npfmt

MX4, MX8 = 0, 1
COVER, FLOOR = 0, 1
BLOCK = 32
_FORMAT = {MX4: (4, 1, 1), MX8: (8, 3, 9)}            # bits, significand bits, -log2 alpha


def magnitudes(elem: int) -> np.ndarray:
    """The non-negative elements in the order of their codes."""
    n, p, f = _FORMAT[elem]
    count = (1 << (n - 1)) - (1 if elem == MX8 else 0)
    return np.array([npfmt.decode(c, n, p) * 2.0 ** -f for c in range(count)])


def scale_byte(amax: float, elem: int, rule: int) -> int:
    """The scale byte of a block with this largest magnitude, by search over the bytes."""
    if not np.isfinite(amax):
        return 255
    top = magnitudes(elem)[-1]
    if rule == COVER:
        return next(s for s in range(255) if amax <= top * 2.0 ** (s - 127))
    low = 2.0 ** np.floor(np.log2(top))
    fits = [s for s in range(255) if low * 2.0 ** (s - 127) <= amax]
    return fits[-1] if fits else 0


def nearest_code(v, elem: int) -> np.ndarray:
    """Code of the nearest element, ties to the even code, saturating; no code of -0."""
    table = magnitudes(elem)
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(v), table[-1])
    up = np.clip(np.searchsorted(table, a), 1, len(table) - 1)          # table[up - 1] < a <= table[up], or the first two
    below, above = a - table[up - 1], table[up] - a
    code = np.where((below < above) | ((below == above) & (up % 2 == 1)), up - 1, up)
    return np.where((v < 0) & (code > 0), code | (8 if elem == MX4 else 128), code).astype(np.uint8)


def quantize(x, elem: int, rule: int):
    """[rows, K] -> (codes as stored, scales padded with zeros to a multiple of four)."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    nb = -(-K // BLOCK)
    full = np.zeros((rows, nb * BLOCK))
    full[:, :K] = x
    blocks = full.reshape(rows, nb, BLOCK)
    scales = np.zeros((rows, -(-nb // 4) * 4), np.uint8)
    codes = np.zeros((rows, nb, BLOCK), np.uint8)
    for r in range(rows):
        for b in range(nb):
            s = scale_byte(np.abs(blocks[r, b]).max(), elem, rule)
            scales[r, b] = s
            if s != 255:
                codes[r, b] = nearest_code(np.ldexp(blocks[r, b], 127 - s), elem)
    codes = codes.reshape(rows, nb * BLOCK)
    return (codes[:, 0::2] | codes[:, 1::2] << 4 if elem == MX4 else codes), scales


def values(codes, scales, elem: int, K: int) -> np.ndarray:
    """What the stored bytes stand for, [rows, K]."""
    codes, scales = np.asarray(codes, np.uint8), np.asarray(scales, np.uint8)
    if elem == MX4:
        codes = np.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)
    table = magnitudes(elem)
    if elem == MX8:
        table = np.append(table, np.nan)
    v = np.concatenate((table, -table))[codes]
    nb = v.shape[1] // BLOCK
    alpha = np.where(scales[:, :nb] == 255, np.nan, 2.0 ** (scales[:, :nb].astype(np.float64) - 127))
    return (v.reshape(-1, nb, BLOCK) * alpha[:, :, None]).reshape(v.shape)[:, :K]


def linear(x, w, bias=None, relu: bool = False) -> np.ndarray:
    """x [M, K], w [N, K] as values."""
    y = x @ w.T + (0 if bias is None else np.asarray(bias, np.float64))
    return np.where(y < 0, 0, y) if relu else y


def rms_norm(x, add, weight, eps: float):
    """(x + add as float32 holds it, the norm of that)."""
    s = np.asarray(x, np.float32) if add is None else np.asarray(x, np.float32) + np.asarray(add, np.float32)
    d = s.astype(np.float64)
    v = d / np.sqrt((d * d).mean(1, keepdims=True) + np.float64(np.float32(eps)))
    return s, v if weight is None else v * np.asarray(weight, np.float64)
