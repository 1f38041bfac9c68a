"""Matrices in 8 bits, their products and the gated feed-forward block restated in numpy and 64 bits from the definitions."""
from __future__ import annotations

from typing import NamedTuple

import numpy as np

BLOCK = 128


class Held(NamedTuple):
    codes: np.ndarray       # uint8 [rows, cols]
    bytes: np.ndarray       # uint8 [rows, blocks]


def _e4m3(v):
    """Codes of |v| <= 448 (fp64), to nearest, ties to even."""
    size = np.abs(v)
    power = np.maximum(np.frexp(size)[1] - 1, -6)                      # size in [2^power, 2^(power + 1)), or below 2^-6
    steps = np.rint(np.ldexp(size, 3 - power)).astype(np.int64)         # 8 .. 16 of 2^(power - 3), 0 .. 8 below 2^-6
    up = steps == 16
    steps, power = np.where(up, 8, steps), np.where(up, power + 1, power)
    code = np.where(steps >= 8, (power + 7) * 8 + steps - 8, steps)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def code_values():
    c = np.arange(128)
    v = np.where(c < 8, c * 2.0 ** -9, np.ldexp(1.0 + (c % 8) / 8, c // 8 - 7))
    v[127] = np.nan
    return np.concatenate([v, -v])


def hold(x) -> Held:
    """fp64 [rows, cols] in 8 bits."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    full = np.zeros((rows, blocks * BLOCK))
    full[:, :cols] = x
    full = full.reshape(rows, blocks, BLOCK)
    broken = ~np.isfinite(full).all(2)
    full = np.where(broken[:, :, None], 0.0, full)
    largest = np.abs(full).max(2) if rows else np.zeros((0, blocks))
    e = np.full(largest.shape, -127)
    some = largest > 0
    e[some] = np.maximum(np.ceil(np.log2(largest[some] / 448.0)).astype(int) - 1, -127)
    for _ in range(3):                                                   # (the logarithm's rounding is mended exactly)
        e = np.where(np.ldexp(448.0, e) < largest, e + 1, e)
    codes = _e4m3(np.ldexp(full, -e[:, :, None]))
    beyond = (e == 120)[:, :, None] & ((codes & 0x7F) == 0x78)            # 256 2^120 is no fp32 number
    codes = np.where(beyond, codes - 1, codes)
    codes = np.where(broken[:, :, None], 0x7F, codes).reshape(rows, -1)[:, :cols]
    return Held(codes.astype(np.uint8), np.where(broken, 255, e + 127).astype(np.uint8))


def values(h: Held):
    rows, cols = h.codes.shape
    e = h.bytes.astype(int) - 127
    power = np.where(h.bytes == 255, np.nan, np.ldexp(1.0, e))
    return code_values()[h.codes] * np.repeat(power, BLOCK, axis=1)[:, :cols]


def scale_index(rows: int, cols: int):
    """Where the byte of every row and block lies."""
    r, b = np.arange(rows)[:, None], np.arange(-(-cols // BLOCK))[None, :]
    return ((b // 4) * (-(-rows // 128)) + r // 128) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def half_step(x):
    """The most by which rounding into 8 bits may move each element of x: half a step of its size, or of the smallest normal one."""
    h = hold(x)
    e = np.repeat(h.bytes.astype(int) - 127, BLOCK, axis=1)[:, :x.shape[1]]
    size = np.maximum(np.abs(x), np.ldexp(1.0, e - 6))
    return np.ldexp(1.0, np.frexp(size)[1] - 1 - 4)


def share(g, gelu: bool):
    y = 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3) if gelu else g
    t = np.exp(-np.abs(y))
    return np.where(y >= 0, 1 / (1 + t), t / (1 + t))


def activation(g, gelu: bool):
    """act(g), act'(g)"""
    s = share(g, gelu)
    dy = 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g ** 2) if gelu else 1.0
    return g * s, s + g * s * share(-g, gelu) * dy
