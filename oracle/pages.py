"""CPU oracle of the paged cache: its layout, the 4-bit format, rotation, and attention over it, in numpy and 64 bits.

TEST INFRASTRUCTURE ONLY; imports nothing from the HIP package.

A page holds 64 rows of K and V of one (sequence, KV head); ``table[u][j]`` is the page of unit u's rows 64 j .. 64 j + 63,
``lens[u]`` its number of rows.  4-bit pages hold, per row and block of 32 dims, a power of two (a byte e for 2^(e - 127)) and a
code of 4 bits per dim: sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Every address is written out for a single element here,
whereas the kernels and the benchmark's plain form move whole pieces.
"""
from __future__ import annotations

import numpy as np

ROWS = 64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def page_bytes(d: int, fp4: bool) -> int:
    return ROWS * d + 2 * ROWS * (d // 32) if fp4 else 2 * ROWS * d * 2


def places(d: int):
    """Byte of (row, dim)'s code in K and V [64, d], and of (row, block)'s scale in K and V [64, d / 32], in a 4-bit page."""
    r, c, b = np.arange(ROWS)[:, None], np.arange(d)[None, :], np.arange(d // 32)[None, :]
    chunk = 4 if d <= 64 else 8 if d <= 128 else 16
    k = r * (d // 2) + c // 2
    v = ROWS * d // 2 + (((r // 4) * (d // chunk) + c // chunk) * 4 + r % 4) * (chunk // 2) + (c % chunk) // 2
    ks = ROWS * d + (b * 16 + r % 16) * 4 + r // 16
    vs = ROWS * d + ROWS * (d // 32) + (((r // 4) % 4 * (d // 32) + b) * 4 + r // 16) * 4 + r % 4
    return k, v, ks, vs


def quantise(x: np.ndarray):
    """Rows x [n, d] (fp64) to codes [n, d] and scale bytes [n, d / 32] (uint8)."""
    n, d = x.shape
    codes, scales = np.zeros((n, d), np.uint8), np.zeros((n, d // 32), np.uint8)
    for i in range(n):
        for b in range(d // 32):
            y = x[i, 32 * b:32 * b + 32]
            if not np.isfinite(y).all():
                scales[i, b] = 255
                continue
            s = -126
            while np.abs(y).max() >= 7.0 * 2.0 ** s:
                s += 1
            scales[i, b] = s + 127
            z = np.abs(y) / 2.0 ** s
            dist = np.abs(z[:, None] - GRID[None, :])
            near = dist.argmin(1)                                       # the lower of two equally near ones
            up = np.minimum(near + 1, 7)
            tie = (dist[np.arange(32), near] == dist[np.arange(32), up]) & (up != near)
            code = np.where(tie & (near % 2 == 1), up, near)
            codes[i, 32 * b:32 * b + 32] = code + 8 * np.signbit(y)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    x = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return x * np.repeat(s, 32, axis=-1)


def rotate(x: np.ndarray, positions: np.ndarray, rope: np.ndarray, halves: bool) -> np.ndarray:
    """x [S, n, heads, d] fp64 by the table rope [n_positions, 2, rot / 2] (fp32 cosines, sines): fp32 values."""
    out = x.astype(np.float64).copy()
    half = rope.shape[-1]
    for i in range(half):
        a, b = (i, i + half) if halves else (2 * i, 2 * i + 1)
        p = np.clip(positions, 0, rope.shape[0] - 1)
        c, s = rope[p, 0, i].astype(np.float64)[..., None], rope[p, 1, i].astype(np.float64)[..., None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out.astype(np.float32).astype(np.float64)


def write_row(page: np.ndarray, row: int, key: bool, x: np.ndarray, fp4: bool, to_bits) -> None:
    """Row of K or V into a page (uint8 [bytes]); to_bits: fp64 -> the 16-bit type's bits (uint16)."""
    d = x.shape[0]
    if not fp4:
        at = (0 if key else ROWS * d * 2) + row * d * 2
        page[at:at + 2 * d] = to_bits(x).view(np.uint8)
        return
    k, v, ks, vs = places(d)
    codes, scales = quantise(x[None])
    at = (k if key else v)[row]
    page[at[0::2]] = codes[0, 0::2] | codes[0, 1::2] << 4               # the dims 2 i and 2 i + 1 share a byte
    page[(ks if key else vs)[row]] = scales[0]


def read_rows(page: np.ndarray, d: int, fp4: bool, from_bits):
    """K and V [64, d] fp64 of a page."""
    if not fp4:
        w = from_bits(page.view(np.uint16)).reshape(2, ROWS, d)
        return w[0], w[1]
    k, v, ks, vs = places(d)
    shift = 4 * (np.arange(d) % 2)
    return tuple(values(page[c] >> shift & 15, page[s]) for c, s in ((k, ks), (v, vs)))


def attention(q: np.ndarray, pool: np.ndarray, table: np.ndarray, lens: np.ndarray, H: int, scale: float, d: int, fp4: bool,
              from_bits):
    """q [S, n, Hq, d] fp64 over pages: (out, lse) fp64.  Token t sees rows before lens - (n - 1 - t) on pages that exist."""
    S, n, Hq, _ = q.shape
    G = Hq // H
    out, lse = np.zeros((S, n, Hq, d)), np.full((S, n, Hq), -np.inf)
    for u in range(S * H):
        s, h = divmod(u, H)
        length = min(max(int(lens[u]), 0), 64 * table.shape[1])
        K, V, there = np.zeros((length, d)), np.zeros((length, d)), np.zeros(length, bool)
        for j in range((length + 63) // 64):
            p = int(table[u, j])
            if 0 <= p < pool.shape[0]:
                k, v = read_rows(pool[p], d, fp4, from_bits)
                m = min(64, length - 64 * j)
                K[64 * j:64 * j + m], V[64 * j:64 * j + m], there[64 * j:64 * j + m] = k[:m], v[:m], True
        for t in range(n):
            see = there & (np.arange(length) < length - (n - 1 - t))
            if not see.any():
                continue
            z = scale * (q[s, t, h * G:(h + 1) * G] @ K[see].T)
            top = z.max(-1, keepdims=True)
            e = np.exp(z - top)
            out[s, t, h * G:(h + 1) * G] = (e / e.sum(-1, keepdims=True)) @ V[see]
            lse[s, t, h * G:(h + 1) * G] = top[:, 0] + np.log(e.sum(-1))
    return out, lse
