"""fp64 restatement of the paged cache held in 4 bits: the format, the pages, the attention over them.

Written from the definitions in include/cachefocus.h with plain loops and Python integers; test infrastructure only."""
from __future__ import annotations

from typing import List, Optional, Tuple

import numpy as np

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 32


def round_to_bf16(x: float) -> float:
    """Nearest number of eight significant bits, ties to even (no limit of range: callers stay inside it)."""
    if x == 0.0:
        return 0.0
    fraction, power = np.frexp(np.float64(x))
    return float(np.ldexp(np.rint(fraction * 256.0), power - 8))


def quantise_group(x: np.ndarray) -> Tuple[List[int], float]:
    """(codes, scale) of a group's numbers."""
    x = np.asarray(x, np.float64)
    if not np.all(np.isfinite(x)):
        return [0] * len(x), float("nan")
    scale = round_to_bf16(float(np.max(np.abs(x))) / 6.0)
    if scale < 2.0 ** -126:
        return [0] * len(x), 0.0
    codes = []
    for value in x:
        best = min(range(8), key=lambda c: (abs(abs(value) - LEVELS[c] * scale), c % 2))
        codes.append(best | (8 if np.signbit(value) else 0))
    return codes, scale


def quantise(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """(codes [..., D], scales [..., D / 32]) of x [..., D]: quantise_group of every group."""
    x = np.asarray(x, np.float64)
    groups = x.reshape(-1, GROUP)
    bad = ~np.isfinite(groups).all(-1)
    groups = np.where(bad[:, None], 0.0, groups)
    fraction, power = np.frexp(np.abs(groups).max(-1) / 6.0)
    scales = np.ldexp(np.rint(fraction * 256.0), power - 8)
    scales[scales < 2.0 ** -126] = 0.0
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])                       # even codes first: they keep a tie
    levels = np.array(LEVELS)[order]
    codes = order[np.argmin(np.abs(np.abs(groups)[..., None] - levels * scales[:, None, None]), -1)] | (8 * np.signbit(groups))
    codes[(scales == 0.0) | bad] = 0
    scales[bad] = np.nan
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1] + (x.shape[-1] // GROUP,))


def numbers(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What codes and scales stand for."""
    level = np.array(LEVELS + tuple(-x for x in LEVELS))[codes]
    with np.errstate(invalid="ignore"):
        return level * np.repeat(scales, GROUP, axis=-1)


def places(head_dim: int) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """Where a block keeps things: (key codes, value codes) as nibble numbers [16, D] (2 * byte + half), (key scales, value
    scales) as byte numbers [16, D / 32]."""
    k, v = np.zeros((16, head_dim), np.int64), np.zeros((16, head_dim), np.int64)
    ks, vs = np.zeros((16, head_dim // GROUP), np.int64), np.zeros((16, head_dim // GROUP), np.int64)
    for row in range(16):
        h, t_row, p = row // 8, row % 8 // 2, row % 2
        for dim in range(head_dim):
            j, rest = divmod(dim, GROUP)
            t, i = divmod(rest, 8)
            k[row, dim] = 2 * (row * (head_dim // 2) + t * (head_dim // 8) + 4 * j + i // 2) + i % 2
            u, i = divmod(rest, 4)
            v[row, dim] = 2 * (8 * head_dim + h * 4 * head_dim + u * (head_dim // 2) + t_row * (head_dim // 8) + p * (head_dim // 16) + 2 * j + i // 2) + i % 2
        for j in range(head_dim // GROUP):
            ks[row, j] = 16 * head_dim + row * (head_dim // 16) + 2 * j
            vs[row, j] = 17 * head_dim + row * (head_dim // 16) + 2 * j
    return k, v, ks, vs


def read_block(block: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """Keys and values [16, D] of a block's bytes [18 D]."""
    head_dim = len(block) // 18
    k, v, ks, vs = places(head_dim)
    nibbles = np.stack([block & 15, block >> 4], -1).reshape(-1).astype(np.int64)

    def bf16(at):
        bits = (block[at].astype(np.uint32) | (block[at + 1].astype(np.uint32) << 8)) << 16
        return bits.view(np.float32).astype(np.float64)

    return numbers(nibbles[k], bf16(ks)), numbers(nibbles[v], bf16(vs))


class Pool:
    """Pages, one request after the other, in Python integers."""

    def __init__(self, n_requests: int, page_rows: int, n_pages: int, cols: int):
        self.page_rows, self.cols = page_rows, cols
        self.table = [[] for _ in range(n_requests)]
        self.rows = [0] * n_requests
        self.free = list(range(n_pages - 1, -1, -1))
        self.status = set()

    def resize(self, rows, extra: int, max_new: Optional[int]) -> List[List[int]]:
        """Slots of the new rows [n_requests][max_new]; RANGE = 2 and WORKSPACE = 4 are added to `status`."""
        targets = []
        for b, r in enumerate(rows):
            target = 0 if r < 0 else int(r) + extra
            if target < 0 or target > self.cols * self.page_rows or (max_new is not None and target - self.rows[b] > max_new):
                self.status.add(2)
                target = None
            targets.append(target)
        for b in reversed(range(len(rows))):
            if targets[b] is not None:
                while len(self.table[b]) > -(-targets[b] // self.page_rows):
                    self.free.append(self.table[b].pop())
        height, asked, slots = len(self.free), 0, []
        for b, target in enumerate(targets):
            old, row_slots = self.rows[b], []
            if target is not None:
                need = max(0, -(-target // self.page_rows) - len(self.table[b]))
                asked += need
                if need and asked > height:
                    self.status.add(4)
                else:
                    self.table[b] += [self.free.pop() for _ in range(need)]
                    self.rows[b] = target
                    row_slots = [self.table[b][r // self.page_rows] * self.page_rows + r % self.page_rows for r in range(old, target)]
            slots.append((row_slots + [-1] * (max_new or 0))[:max_new or 0])
        return slots


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """q [n, Hq, D], the last n rows of k, v [rows, Hkv, D] being the queries' own: (out [n, Hq, D], lse [Hq, n], sum of p |v|
    [n, Hq, D], largest sum of |q k| scale [n, Hq])."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((heads, n), -np.inf), np.zeros((n, heads))
    for j in range(n):
        sees = k.shape[0] - n + j + 1
        if sees <= 0:
            continue
        for h in range(heads):
            keys, values = k[:sees, h // group], v[:sees, h // group]
            x = keys @ q[j, h].astype(np.float64) * scale
            top = np.max(x)
            p = np.exp(x - top)
            lse[h, j] = top + np.log(p.sum())
            out[j, h] = p @ values / p.sum()
            spread[j, h] = p @ np.abs(values) / p.sum()
            reach[j, h] = np.max(np.abs(keys) @ np.abs(q[j, h].astype(np.float64))) * abs(scale)
    return out, lse, spread, reach
