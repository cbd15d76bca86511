"""The 8-bit KV cache in float64 numpy: codes, block order, tail and attention.

Written from the definitions in include/dv.h, number by number: a cache here is a
list of rows per (layer, head), quantised in blocks of 32 as they become whole.
"""
from __future__ import annotations

import numpy as np

BLOCK, TAIL = 32, 96
TOP = {"i8": 127.0, "f8": 448.0}


def e4m3_values() -> np.ndarray:
    """The number of each e4m3 code (0x7f and 0xff are NaN)."""
    code = np.arange(256)
    sign, e, m = np.where(code & 0x80, -1.0, 1.0), code >> 3 & 15, code & 7
    v = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))
    return np.where(code & 0x7f == 0x7f, np.nan, sign * v)


_E4M3 = e4m3_values()


def e4m3_code(y) -> np.ndarray:
    """Nearest code of finite |y| <= 464, ties to the even code."""
    y = np.asarray(y, dtype=np.float64)
    pos = _E4M3[:0x7f]
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(pos, a), 1, 0x7e)
    below, above = a - pos[hi - 1], pos[hi] - a
    code = np.where((below < above) | ((below == above) & ((hi - 1) % 2 == 0)), hi - 1, hi)
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def k_byte(hd: int) -> np.ndarray:
    """Byte of (slot, dim) in a K block, [32][hd]."""
    s, j = np.arange(BLOCK)[:, None], np.arange(hd)[None]
    return ((2 * (j // 64) + s // 4 % 2) * 64 + 16 * (j % 32 // 8) + 4 * (s // 8) + s % 4) * 16 + 8 * (j % 64 // 32) + j % 8


def v_byte(hd: int) -> np.ndarray:
    s, j = np.arange(BLOCK)[:, None], np.arange(hd)[None]
    return (64 * (j // 32) + 16 * (s // 8) + j % 16) * 16 + 8 * (j % 32 // 16) + s % 8


def quantise(x, fmt: str):
    """Codes (uint8 bytes) and fp32 scale of one block of bf16 numbers."""
    x = np.asarray(x, dtype=np.float64)
    top = TOP[fmt]
    if not np.isfinite(x).all():
        return np.zeros(x.shape, np.uint8), np.float32(np.nan)
    most = np.abs(x).max()
    if most < 2.0 ** -100:
        return np.zeros(x.shape, np.uint8), np.float32(0)
    # quotients of fp32 numbers rounded through fp64 are correctly rounded (53 >= 2 24 + 2)
    scale, inv = np.float32(most / top), np.float32(top / most)
    y = (x * np.float64(inv)).astype(np.float32)  # the product is exact in fp64
    if fmt == "i8":
        return np.rint(y).astype(np.int8).view(np.uint8), scale
    return e4m3_code(y), scale


def numbers(codes, fmt: str) -> np.ndarray:
    codes = np.asarray(codes).view(np.uint8)
    return codes.view(np.int8).astype(np.float64) if fmt == "i8" else _E4M3[codes]


class Cache:
    """K or V of one (layer, head): rows as floats that bf16 holds, blocks of codes
    in row order [32][hd]."""

    def __init__(self, hd: int, fmt: str):
        self.hd, self.fmt = hd, fmt
        self.blocks = []                       # (codes, scale)
        self.tail = np.zeros((0, hd))

    def __len__(self):
        return BLOCK * len(self.blocks) + len(self.tail)

    def append(self, rows):
        rows = np.concatenate([self.tail, np.asarray(rows, dtype=np.float64).reshape(-1, self.hd)])
        while len(rows) >= BLOCK:
            self.blocks.append(quantise(rows[:BLOCK], self.fmt))
            rows = rows[BLOCK:]
        self.tail = rows

    def rows(self) -> np.ndarray:
        """What attention sees, [len][hd]."""
        parts = [numbers(c, self.fmt) * np.float64(s) for c, s in self.blocks] + [self.tail]
        return np.concatenate(parts)


def attention(q, k, v, sees):
    """q [n][hd], k and v [keys][hd], sees bool [n][keys]: softmax attention, zeros
    for a row that sees nothing.  Numbers of keys that a row does not see do not enter
    it, whatever they are."""
    out = np.zeros(q.shape)
    for i in range(len(q)):
        at = np.flatnonzero(sees[i])
        if len(at):
            z = k[at] @ q[i] / np.sqrt(q.shape[1])
            w = np.exp(z - z.max())
            out[i] = (w / w.sum()) @ v[at]
    return out
