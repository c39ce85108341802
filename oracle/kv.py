"""Definitions of the key/value cache in four bits in float64, for the tests: block tables, the four-bit values, norm and rotation
of heads, attention.  Written from the formulas; shares nothing with the library."""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

BLOCK = 64
GROUP = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


class BlockTables:
    """Rows of blocks over a pool; the lowest free blocks go first."""

    def __init__(self, n_blocks: int, max_seqs: int, max_seq_tokens: int):
        self.n_blocks, self.max_seqs, self.max_seq_tokens = n_blocks, max_seqs, max_seq_tokens
        self.row_blocks = -(-max_seq_tokens // BLOCK)
        self.rows: List[List[int]] = [[] for _ in range(max_seqs)]
        self.free = set(range(n_blocks))
        self.refused = self.exhausted = False

    def extend(self, seq, length, new, T: int, max_new: int):
        """(start, position, slot) of the step, the latter two -1 where a request is refused."""
        start, position, slot = [0], [-1] * T, [-1] * T
        first = 0
        accepted, need_before, free = [], 0, sorted(self.free)
        for i, (r, l, a) in enumerate(zip(seq, length, new)):
            rows = max(0, a)
            ok = (0 <= r < self.max_seqs and r not in seq[:i] and l >= 0 and 0 <= a <= min(max_new, T) and l + a <= self.max_seq_tokens
                  and -(-l // BLOCK) <= len(self.rows[r]) and first + rows <= T)
            if not ok:
                self.refused = True
            else:
                need = max(0, -(-(l + a) // BLOCK) - len(self.rows[r]))
                if need and need_before + need > len(free):
                    self.exhausted = True
                else:
                    accepted.append((i, r, l, a, first, free[need_before:need_before + need]))
                need_before += need
            first += rows
            start.append(min(first, T))
        for i, r, l, a, at, blocks in accepted:
            self.rows[r] += blocks
            self.free -= set(blocks)
            for j in range(a):
                position[at + j] = l + j
                slot[at + j] = self.rows[r][(l + j) // BLOCK] * BLOCK + (l + j) % BLOCK
        return start, position, slot

    def release(self, seq, keep: Optional[Sequence[int]] = None):
        for i, r in enumerate(seq):
            k = 0 if keep is None else keep[i]
            if not 0 <= r < self.max_seqs or k < 0:
                self.refused = True
                continue
            n = -(-k // BLOCK)
            self.free |= set(self.rows[r][n:])
            del self.rows[r][n:]

    def table(self) -> np.ndarray:
        return np.array([row + [-1] * (self.row_blocks - len(row)) for row in self.rows], dtype=np.int32)


def four_bits(x: np.ndarray) -> np.ndarray:
    """The values that the cache holds for float64 x [..., multiple of 32] (NaN: 0, infinities: the largest)."""
    out = np.empty(x.size)
    for i, g in enumerate(np.where(np.isnan(x), 0.0, x).reshape(-1, GROUP)):
        top = np.abs(g).max()
        e = -100
        while top > 7.0 * 2.0 ** e and e < 125:
            e += 1
        # nearest magnitude, ties to the even code: the borders half way between neighbours
        y = np.abs(g) / 2.0 ** e
        code = np.zeros(GROUP, dtype=int)
        for c in range(1, 8):
            border = (MAGNITUDES[c - 1] + MAGNITUDES[c]) / 2
            code[(y >= border) if c % 2 == 0 else (y > border)] = c
        out[i * GROUP:(i + 1) * GROUP] = np.copysign(MAGNITUDES[code] * 2.0 ** e, g)
    return out.reshape(x.shape)


def norm_rotate(x: np.ndarray, weight: Optional[np.ndarray], eps: float, position: np.ndarray, inv_freq: Optional[np.ndarray],
                neighbours: bool = False) -> np.ndarray:
    """x [T, heads, dim] float64."""
    u = x.astype(np.float64)
    if weight is not None:
        u = u / np.sqrt(np.mean(u * u, axis=-1, keepdims=True) + eps) * weight
    if inv_freq is None:
        return u
    a = np.asarray(position, dtype=np.float64)[:, None, None] * inv_freq.astype(np.float64)
    c, s = np.cos(a), np.sin(a)
    half = x.shape[-1] // 2
    first = np.s_[..., 0::2] if neighbours else np.s_[..., :half]
    second = np.s_[..., 1::2] if neighbours else np.s_[..., half:]
    y = np.empty_like(u)
    y[first] = u[first] * c - u[second] * s
    y[second] = u[second] * c + u[first] * s
    return y


def attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray, length: int, scale: float) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """q [n, heads, dim], keys / values [length + n, kv heads, dim] float64 -> (out, sum of weights * |values|, largest
    sum |q k| * |scale|), the latter two for error bounds."""
    n, h, d = q.shape
    group = h // keys.shape[1]
    out, size, top = np.zeros_like(q), np.zeros_like(q), np.zeros((n, h, 1))
    for i in range(h):
        k, v = keys[:, i // group], values[:, i // group]
        s = scale * (q[:, i] @ k.T)
        hidden = np.arange(length + n)[None] > np.arange(length, length + n)[:, None]
        s[hidden] = -math.inf
        with np.errstate(invalid="ignore"):
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
        out[:, i], size[:, i] = p @ v, p @ np.abs(v)
        top[:, i, 0] = abs(scale) * np.max(np.where(hidden, 0.0, np.abs(q[:, i]) @ np.abs(k).T), axis=1)
    return out, size, top
