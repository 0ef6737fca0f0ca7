"""Float64 reference of what lies between two projections of a decoder layer: root-mean-square norm, rotary positions, and
attention over rows that a page table names.  Plain numpy, one loop per sequence and head, written from the formulas."""
from __future__ import annotations

import math

import numpy as np


def rms_norm(x: np.ndarray, gamma: np.ndarray, eps: float, residual: np.ndarray | None = None):
    """(h, y): h = x + residual, y = h / sqrt(mean h^2 + eps) * gamma, row by row."""
    h = x.astype(np.float64) if residual is None else x.astype(np.float64) + residual.astype(np.float64)
    y = np.empty_like(h)
    for i, row in enumerate(h):
        y[i] = row / math.sqrt(float(np.dot(row, row)) / row.size + eps) * gamma.astype(np.float64)
    return h, y


def rope_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, trained: float = 0.0, low: float = 1.0, high: float = 4.0) -> np.ndarray:
    """Angle per position of every pair.  trained > 0: a wave that turns more than `high` times over the trained length stays, one of fewer
    than `low` turns is stretched by `factor`, those between in proportion; trained = 0: all are stretched."""
    w = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    out = []
    for f in w:
        keep = 0.0
        if trained > 0:
            turns = trained / (2 * math.pi / f)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
        out.append(f * (keep + (1 - keep) / factor))
    return np.array(out)


def rotate(x: np.ndarray, angles: np.ndarray, pairs: bool) -> np.ndarray:
    """x: heads x width of one row; angles: rot / 2.  Components (i, i + rot / 2), or with `pairs` (2 i, 2 i + 1), turn by angle i."""
    n = angles.size
    first = np.arange(n) * 2 if pairs else np.arange(n)
    second = first + 1 if pairs else first + n
    out = x.astype(np.float64).copy()
    z = (out[:, first] + 1j * out[:, second]) * np.exp(1j * angles)
    out[:, first], out[:, second] = z.real, z.imag
    return out


def cache_rows(cache: np.ndarray, pages: np.ndarray, head: int, count: int) -> np.ndarray:
    """The first `count` rows of a sequence: cache is pages x heads x rows x width."""
    size = cache.shape[2]
    return np.array([cache[pages[p // size], head, p % size] for p in range(count)], dtype=np.float64).reshape(count, cache.shape[3])


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float, seen: int):
    """(softmax(scale q k^T) v, softmax(...) |v|) of one query over the first `seen` rows; zeros where there are none."""
    if seen <= 0:
        return np.zeros(v.shape[1]), np.zeros(v.shape[1])
    s = k[:seen] @ q.astype(np.float64) * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ v[:seen], w @ np.abs(v[:seen])


def attention(Q: np.ndarray, K: np.ndarray, V: np.ndarray, n_q_heads: int, row_start, kv_len, page_table: np.ndarray, scale: float, causal: bool):
    """(O, the same with |v| in place of v) of all rows.  Q: rows x heads * width; K, V: pages x heads x rows x width."""
    d, hkv = K.shape[3], K.shape[1]
    O, A = np.zeros(Q.shape), np.zeros(Q.shape)
    for s in range(len(kv_len)):
        n = row_start[s + 1] - row_start[s]
        for g in range(hkv):
            k, v = (cache_rows(c, page_table[s], g, int(kv_len[s])) for c in (K, V))
            for h in range(g * n_q_heads // hkv, (g + 1) * n_q_heads // hkv):
                for j in range(n):
                    row = row_start[s] + j
                    seen = int(kv_len[s]) - n + j + 1 if causal else int(kv_len[s])
                    O[row, h * d:(h + 1) * d], A[row, h * d:(h + 1) * d] = attend(Q[row, h * d:(h + 1) * d], k, v, scale, seen)
    return O, A
