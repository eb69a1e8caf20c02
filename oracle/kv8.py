"""Oracle of the position rotation and of the 8-bit cache, in 64 bits.  Test infrastructure only: plain loops over
requests and blocks, rounding by search among all e4m3 numbers, tiles addressed byte by byte from the formulas of the pool's layout.

A block's scale is 2^(s-127): s - 127 is the smallest integer e with amax <= 448 * 2^e over the finite values that join the
block (s at least 1), and with tokens that the block already holds the larger of theirs and that.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
NAN = 0x7F


def _values() -> np.ndarray:
    got = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if (e, m) == (15, 7) else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0**-6
        got.append(-v if c & 128 else v)
    return np.asarray(got)


VALUES = _values()


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 codes of |x| <= 448, ties to the even code; NaN and infinities give NaN."""
    grid = VALUES[:127]
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0)
    hi = np.minimum(np.searchsorted(grid, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo) | np.where(np.signbit(x), 128, 0)
    return np.where(fine, code, NAN).astype(np.uint8)


def scale_byte(amax: float) -> int:
    s = 1
    while amax > math.ldexp(448.0, s - 127):
        s += 1
    return s


def byte_of(d: int, is_k: bool) -> np.ndarray:
    """[16, d]: byte of a tile that holds element e of token t."""
    t, e = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    return (e // 16 * 16 + t) * 16 + e % 16 if is_k else (((e // 64 * 4 + t // 4) * 16 + e % 16) * 4 + e % 64 // 16) * 4 + t % 4


def block_bytes(heads: int, d: int) -> int:
    return heads * BLOCK * d + (heads + 15) // 16 * 16


def read_tokens(plane: np.ndarray, table_row, length: int, heads: int, d: int, is_k: bool) -> np.ndarray:
    """plane [blocks, bytes] -> the first `length` tokens of a request, [length, heads, d] float64."""
    at = byte_of(d, is_k)
    out = np.empty((length, heads, d))
    for j0 in range(0, length, BLOCK):
        b = plane[int(table_row[j0 // BLOCK])]
        n = min(BLOCK, length - j0)
        for h in range(heads):
            s = int(b[heads * BLOCK * d + h])
            out[j0:j0 + n, h] = np.ldexp(VALUES[b[h * BLOCK * d:(h + 1) * BLOCK * d][at]], s - 127)[:n]
    return out


def write_tokens(plane: np.ndarray, table_row, first: int, x: np.ndarray, is_k: bool) -> None:
    """In place: x [n, heads, d] becomes tokens first .. first + n - 1 of a request."""
    n, heads, d = x.shape
    at = byte_of(d, is_k)
    pos = first
    while pos < first + n:
        have = pos % BLOCK if pos == first else 0
        count = min(BLOCK - have, first + n - pos)
        b = plane[int(table_row[pos // BLOCK])]
        rows = x[pos - first:pos - first + count]
        for h in range(heads):
            tile, sat = b[h * BLOCK * d:(h + 1) * BLOCK * d], heads * BLOCK * d + h
            v = rows[:, h]
            fine = np.abs(v[np.isfinite(v)])
            s = scale_byte(float(fine.max()) if fine.size else 0.0)
            if have:
                old = int(b[sat])
                s = max(s, old)
                if s != old:
                    tile[at[:have]] = encode(np.ldexp(VALUES[tile[at[:have]]], old - s))
            tile[at[have:have + count]] = encode(np.ldexp(v, 127 - s))
            b[sat] = s
        pos += count


def rotate(x: np.ndarray, first: int, cos_sin: np.ndarray, interleaved: bool) -> np.ndarray:
    """x [n, heads, d] of positions first .. first + n - 1; cos_sin [positions, rot_dim] fp32."""
    rot = cos_sin.shape[1]
    out = np.array(x, np.float64)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = (cos_sin[first:first + len(x), j].astype(np.float64)[:, None] for j in (i, i + rot // 2))
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return out


def angles(positions: int, rot_dim: int, base: float = 10000.0) -> np.ndarray:
    a = np.arange(positions)[:, None] * base ** (-np.arange(0, rot_dim, 2) / rot_dim)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
