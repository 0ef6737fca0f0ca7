"""Float64 reference of what a server of many tenants adds to a layer: blocks of 4 bits and how a paged cache of them is laid out, and low-rank
adapters row by row.  Plain numpy, written from the definitions."""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def hold_block(x: np.ndarray):
    """(codes 0 ... 15, scale byte) of 32 values: by search over all scales and all levels."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(BLOCK, dtype=np.uint8), 255
    top = np.abs(x).max()
    e = next((e for e in range(-110, 126) if top <= 7 * 2.0 ** e), 125)
    codes = np.zeros(BLOCK, dtype=np.uint8)
    for i, v in enumerate(x):
        far = np.abs(np.abs(v) / 2.0 ** e - LEVELS)
        near = np.flatnonzero(far == far.min())
        best = near[0] if len(near) == 1 else next(k for k in near if k % 2 == 0)
        codes[i] = best + (8 if np.signbit(v) else 0)
    return codes, e + 127


def hold(x: np.ndarray):
    """(codes, scale bytes) of rows whose width is whole blocks: the same by borders, for many values at once."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    bad = ~np.isfinite(blocks).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(bad[..., None], 0.0, blocks)).max(-1))
    f, k = np.frexp(top)
    e = np.clip(np.where(top == 0, -110, np.where(f <= 0.875, k - 3, k - 2)), -110, 125)
    size = np.abs(np.where(bad[..., None], 0.0, blocks)) / np.exp2(e.astype(np.float64))[..., None]
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    for i in range(7):
        middle = (LEVELS[i] + LEVELS[i + 1]) / 2
        codes += (size >= middle if i % 2 else size > middle).astype(np.uint8)
    codes += np.where(np.signbit(blocks) & ~bad[..., None], 8, 0).astype(np.uint8)
    return codes.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def held(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values that codes and scale bytes stand for."""
    size = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (size.reshape(*scales.shape, BLOCK) * s[..., None]).reshape(codes.shape)


def piece_bytes(page_rows: int, d: int) -> int:
    return page_rows * (d // 2 + d // BLOCK)


def code_byte(page_rows: int, d: int, row: int, byte: int, values: bool) -> int:
    """Where in a head's piece of a page byte `byte` of a row's codes lies."""
    if not values:
        return row * (d // 2) + byte
    unit = d // 32
    return row // 4 * (2 * d) + byte // unit * 4 * unit + row % 4 * unit + byte % unit


def scale_byte(page_rows: int, d: int, row: int, block: int, values: bool) -> int:
    first, per = page_rows * d // 2, d // BLOCK
    return first + row // 4 * 4 * per + 4 * block + row % 4 if values else first + row * per + block


def places(page_rows: int, d: int, values: bool):
    """(rows x d / 2, rows x d / 32) places of all bytes of a piece."""
    return (np.array([[code_byte(page_rows, d, r, b, values) for b in range(d // 2)] for r in range(page_rows)]),
            np.array([[scale_byte(page_rows, d, r, b, values) for b in range(d // BLOCK)] for r in range(page_rows)]))


def pack(codes: np.ndarray, scales: np.ndarray, values: bool) -> np.ndarray:
    """(pages, heads, rows, d) codes and their scale bytes -> (pages, heads, bytes)."""
    rows, d = codes.shape[2:]
    out = np.zeros((*codes.shape[:2], piece_bytes(rows, d)), dtype=np.uint8)
    at, at_scale = places(rows, d, values)
    out[:, :, at] = codes[..., 0::2] | codes[..., 1::2] << 4
    out[:, :, at_scale] = scales
    return out


def unpack(pieces: np.ndarray, rows: int, d: int, values: bool) -> np.ndarray:
    """(pages, heads, bytes) -> (pages, heads, rows, d) values."""
    at, at_scale = places(rows, d, values)
    pair = pieces[:, :, at]
    codes = np.stack((pair & 15, pair >> 4), -1).reshape(*pieces.shape[:2], rows, d)
    return held(codes, pieces[:, :, at_scale])


def adapt(H, base, A, B, scale, which, part_ends):
    """(Z, the same with the sizes of all terms): A adapters x (parts x rank) x d, B adapters x columns x rank."""
    rank = B.shape[2]
    Z, size = base.astype(np.float64).copy(), np.abs(base).astype(np.float64)
    for i, w in enumerate(which):
        if not 0 <= w < A.shape[0]:
            continue
        begin = 0
        for k, end in enumerate(part_ends):
            a = A[w, k * rank:(k + 1) * rank].astype(np.float64)
            b = B[w, begin:end].astype(np.float64)
            Z[i, begin:end] += scale[w] * (b @ (a @ H[i]))
            size[i, begin:end] += abs(scale[w]) * (np.abs(b) @ (np.abs(a) @ np.abs(H[i])))
            begin = end
    return Z, size
