"""The 8-bit paged cache in plain numpy: codes and scales, block tables, appending, compaction and
attention, from the definitions in include/kvevict.h, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Codes are uint8 arrays of bit patterns (e4m3: sign, 4 exponent bits with bias 7, 3 mantissa bits, 0x7F
and 0xFF not numbers; int8: two's complement).
"""
from __future__ import annotations

from typing import Optional

import numpy as np

QMAX = {"e4m3": 448.0, "int8": 127.0}


def values(codes: np.ndarray, qtype: str) -> np.ndarray:
    """What the codes stand for, in units of the scale."""
    codes = np.asarray(codes, dtype=np.uint8)
    if qtype == "int8":
        return codes.view(np.int8).astype(np.float64)
    u = np.arange(256)
    e, f = (u >> 3) & 15, (u & 7) / 8.0
    table = np.where(e > 0, (1 + f) * 2.0 ** (e - 7), f * 2.0 ** -6) * np.where(u >= 128, -1.0, 1.0)
    table[[0x7F, 0xFF]] = np.nan
    return table[codes]


def least_scale(amax: float, qtype: str) -> float:
    """The least power of two s >= 2^-126 with amax <= qmax s; 0 for 0."""
    if amax == 0:
        return 0.0
    e = -126
    while amax > QMAX[qtype] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x: np.ndarray, scale: float, qtype: str) -> np.ndarray:
    """x / scale to the nearest code, ties to the even one."""
    # a scale of 0: no finite value but 0, infinities take the largest code all the same
    y = np.asarray(x, dtype=np.float64) / (scale if scale > 0 else 1.0)
    nan = np.isnan(y)
    y = np.where(nan, 0.0, np.clip(y, -QMAX[qtype], QMAX[qtype]))
    if qtype == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    grid = values(np.arange(0x7F), "e4m3")  # the non-negative numbers in order, codes 0 .. 0x7E
    a = np.abs(y)
    hi = np.minimum(np.searchsorted(grid, a), 0x7E)
    lo = np.maximum(hi - 1, 0)
    up = (a - grid[lo] > grid[hi] - a) | ((a - grid[lo] == grid[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8)
    code = np.where(np.signbit(y), code | 0x80, code)
    return np.where(nan, 0x7F, code).astype(np.uint8)


def finite_max(x: np.ndarray) -> float:
    a = np.abs(x[np.isfinite(x)])
    return float(a.max()) if a.size else 0.0


def tables(table: np.ndarray, n_blocks: int, R: int, len_in, add, free, taken: int, n_slots: int):
    """-> (table, len, tok_off, blk_off, slots) after kv_paged_tables."""
    table = table.copy()
    n, stride = table.shape
    tok_off, blk_off, slots, lens = [0], [taken], np.full(n_slots, -1, np.int32), []
    for p in range(n):
        old, new = int(len_in[p]), int(add[p])
        have = min(-(-old // R), stride)
        need = min(-(-(old + new) // R), stride)
        for j in range(have, need):
            at = blk_off[p] + j - have
            b = int(free[at]) if 0 <= at < len(free) else -1
            table[p, j] = b if 0 <= b < n_blocks else -1
        for i in range(new):
            r, t = old + i, tok_off[p] + i
            if t < n_slots and r // R < stride:
                b = int(table[p, r // R])
                slots[t] = b * R + r % R if 0 <= b < n_blocks else -1
        tok_off.append(tok_off[p] + new)
        blk_off.append(blk_off[p] + need - have)
        lens.append(old + new)
    return table, np.array(lens), np.array(tok_off), np.array(blk_off), slots


def append(codes: np.ndarray, scale: np.ndarray, new: np.ndarray, slots: np.ndarray, qtype: str):
    """codes [n_blocks, h_kv, R, d], scale [n_blocks, h_kv], new [T, h_kv, d] (float64), in place."""
    n_blocks, h_kv, R, _ = codes.shape
    t = 0
    while t < len(slots):
        s = int(slots[t])
        if not 0 <= s < n_blocks * R:
            t += 1
            continue
        b, r0, n = s // R, s % R, 1
        while t + n < len(slots) and r0 + n < R and slots[t + n] == s + n:
            n += 1
        for g in range(h_kv):
            rows = new[t:t + n, g]
            was = float(scale[b, g]) if r0 else 0.0
            to = max(was, least_scale(finite_max(rows), qtype))
            if r0 and to > was:
                codes[b, g, :r0] = encode(values(codes[b, g, :r0], qtype) * was, to, qtype)
            codes[b, g, r0:r0 + n] = encode(rows, to, qtype)
            scale[b, g] = to
        t += n


def compact(codes: np.ndarray, scale: np.ndarray, table: np.ndarray, x: np.ndarray, sel: np.ndarray, tail: int,
            qtype: str) -> None:
    """One problem: x [h_kv, L, d] (float64), sel [h_kv, B]; its table's blocks in place."""
    n_blocks, h_kv, R, _ = codes.shape
    L = x.shape[1]
    for g in range(h_kv):
        pos = np.concatenate([np.sort(sel[g]), np.arange(L - tail, L)])
        rows = np.where(((pos >= 0) & (pos < L))[:, None], x[g, np.clip(pos, 0, L - 1)], 0.0)
        for j in range(-(-len(rows) // R)):
            b = int(table[j])
            if not 0 <= b < n_blocks:
                continue
            part = rows[j * R:(j + 1) * R]
            scale[b, g] = least_scale(finite_max(part), qtype)
            codes[b, g, :len(part)] = encode(part, float(scale[b, g]), qtype)


def cache_rows(codes: np.ndarray, scale: np.ndarray, table: np.ndarray, n: int, qtype: str):
    """-> rows 0 .. n - 1 of one problem [h_kv, n, d], and which of them have a block [n]."""
    n_blocks, h_kv, R, d = codes.shape
    ids = np.asarray(table[:-(-n // R)] if n else [], dtype=np.int64)
    ok = (ids >= 0) & (ids < n_blocks)
    at = np.where(ok, ids, 0)
    x = values(codes[at], qtype) * scale[at].astype(np.float64)[..., None, None]
    x = x.transpose(1, 0, 2, 3).reshape(h_kv, -1, d)[:, :n]
    return x, np.repeat(ok, R)[:n]


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, has: np.ndarray, scale: float, length: int,
              cap: Optional[int] = None):
    """q [n, h_q, d] (the last n of `length` rows), k, v [h_kv, rows, d], has [rows].
    -> out [n, h_q, d], and per output the sum of its weights times |v| and its largest sum of |q k| (the
    scales of rounding errors)."""
    n, h_q, d = q.shape
    h_kv, rows = k.shape[:2]
    G = h_q // h_kv
    out, mag, qk = np.zeros((n, h_q, d)), np.zeros((n, h_q, d)), np.zeros((n, h_q, 1))
    for j in range(n):
        seen = np.flatnonzero((np.arange(rows) <= length - n + j) & has)
        if seen.size == 0:
            continue
        for h in range(h_q):
            g = h // G
            t = scale * (k[g, seen] @ q[j, h])
            w = np.exp(t - np.max(t))
            w /= w.sum()
            out[j, h], mag[j, h] = w @ v[g, seen], w @ np.abs(v[g, seen])
            qk[j, h] = abs(scale) * np.max(np.abs(k[g, seen]) @ np.abs(q[j, h]))
    return out, mag, qk
