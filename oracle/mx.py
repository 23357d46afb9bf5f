"""Rows in 8 and 4 bits, their moving average, weight gradient and product, in float64.

Blocks of 32 neighbouring elements of a row share a scale 2^(s - 127), s a byte (255: the block is NaN).
Elements: "int8" an integer q in -127 .. 127 for q / 64; "fp4" a sign and one of GRID.

Quantising a block, step by step as the definition has it: s is the smallest byte for which the block's
largest magnitude, divided by the scale, rounds to at most 127 / 64 (6); at most 254 (252).  Elements round to
the nearest value that the format has, ties to the even q (the even place in the grid); what is larger than
the largest becomes that.  A block that holds a NaN or an infinity is NaN, with elements 0.

Pinned by: a search over all scales, distances to every representable value, a table of hand-made blocks,
central differences of the product (tests).
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TOP_SCALE = {"int8": 254, "fp4": 252}


def blocks(cols: int) -> int:
    return -(-cols // BLOCK)


def _rounds_within(top, s, fmt):
    """Whether a magnitude in units of 2^(s - 127) rounds to no more than the largest element (ties to even: 127.5
    would round to 128, and 7, halfway between 6 and 8, to 8)."""
    u = np.ldexp(top, 127 - s)
    return np.rint(64.0 * u) <= 127.0 if fmt == "int8" else u < 7.0


def scale_bytes(top, fmt):
    """The scales of blocks of largest magnitude ``top`` (finite)."""
    top = np.asarray(top, np.float64)
    s = np.full(top.shape, TOP_SCALE[fmt], np.int64)
    for b in range(TOP_SCALE[fmt] - 1, -1, -1):
        s = np.where(_rounds_within(top, b, fmt), b, s)
    return s


def round_fp4(u):
    """The place in GRID of the nearest value to u >= 0."""
    mid = (GRID[1:] + GRID[:-1]) / 2
    place = np.searchsorted(mid, u, side="left")                # at a tie the lower place
    tie = (place < 7) & (mid[np.minimum(place, 6)] == u)
    return np.where(tie & (place % 2 == 1), place + 1, place)


def quantize(x: np.ndarray, fmt: str):
    """(codes [rows, blocks * 32], scales [rows, blocks]) of the rows of x: q as a signed number, or the 4-bit code."""
    rows, cols = x.shape
    nb = blocks(cols)
    v = np.zeros((rows, nb * BLOCK))
    v[:, :cols] = x
    v = v.reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v)
    s = scale_bytes(np.abs(v).max(axis=2, initial=0.0), fmt)
    u = np.ldexp(v, (127 - s)[:, :, None])
    if fmt == "int8":
        code = np.clip(np.rint(64.0 * u), -127, 127).astype(np.int64)
    else:
        code = np.minimum(round_fp4(np.abs(u)), 7) + 8 * np.signbit(u)
    code = np.where(bad[:, :, None], 0, code)
    return code.reshape(rows, nb * BLOCK), np.where(bad, 255, s)


def values(code: np.ndarray, s: np.ndarray, cols: int, fmt: str) -> np.ndarray:
    """What codes and scales stand for, [rows, cols]."""
    code, s = np.asarray(code, np.int64), np.asarray(s, np.int64)
    if fmt == "int8":
        v = code / 64.0
    else:
        v = np.where(code >= 8, -GRID[code % 8], GRID[code % 8])
    scale = np.where(s == 255, np.nan, np.ldexp(1.0, np.minimum(s, 254) - 127))
    return (v * np.repeat(scale, BLOCK, axis=1))[:, :cols]


def to_bytes(code: np.ndarray, fmt: str) -> np.ndarray:
    """Codes as they are held: a byte each, or two to a byte, the even element in the low half."""
    if fmt == "int8":
        return code.astype(np.int8).view(np.uint8)
    return (code[:, 0::2] + 16 * code[:, 1::2]).astype(np.uint8)


def from_bytes(Q: np.ndarray, fmt: str) -> np.ndarray:
    if fmt == "int8":
        return Q.view(np.int8).astype(np.int64)
    return np.stack((Q % 16, Q // 16), axis=2).reshape(len(Q), -1).astype(np.int64)


def gather(x: np.ndarray, index) -> np.ndarray:
    """Rows of x by index: negative ones are zeros, those past the end NaN."""
    out = np.zeros((len(index), x.shape[1]))
    for k, i in enumerate(index):
        if 0 <= i < len(x):
            out[k] = x[i]
        elif i >= len(x):
            out[k] = np.nan
    return out


def average(state: np.ndarray, v: np.ndarray, gamma: float) -> np.ndarray:
    return gamma * state + (1.0 - gamma) * v


def wgrad(v: np.ndarray, J: np.ndarray, H=None) -> np.ndarray:
    """dW = v^T (J o 1[H > 0])."""
    return v.T @ (J if H is None else np.where(H > 0, J, 0.0))


def product(a: np.ndarray, b: np.ndarray, relu: bool = False) -> np.ndarray:
    c = a @ b.T
    return np.where(c < 0, 0.0, c) if relu else c
