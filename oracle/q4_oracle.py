"""The paged 4-bit cache in plain numpy and Python, 64 bits, row by row and
page by page: what the kernels are checked against.  Shares no code with them.
"""

from __future__ import annotations

import numpy as np

GROUP = 32
TILE = 16


def quantise(x: np.ndarray):
    """fp64 rows [..., d] (bf16 values) -> codes (-7 .. 7) and scales [..., d / 32]."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    with np.errstate(all="ignore"):
        m = np.abs(g).max(-1)
        bad = ~np.isfinite(m)
        mant, e = np.frexp(np.where(bad, 0.0, m) / 7.0)
        s = np.ldexp(np.round(mant * 256.0) / 256.0, e)         # eight bits, ties to even
        s = np.where(s < 2.0 ** -126, 0.0, s)
        code = np.floor(g / np.where(s > 0, s, 1.0)[..., None] + 0.5)
    code = np.where((s > 0)[..., None] & ~bad[..., None], code, 0.0)
    return code.astype(np.int64).reshape(x.shape), np.where(bad, np.nan, s)


def values(x: np.ndarray) -> np.ndarray:
    code, s = quantise(x)
    return code * np.repeat(s, GROUP, -1)


def scale_bits(s: np.ndarray) -> np.ndarray:
    """bf16 bits of scales that bf16 holds exactly."""
    bits = (np.asarray(s, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.where(np.isnan(s), np.uint16(0x7FC0), bits)


def write_row(rec: np.ndarray, row: int, k, v, empty: bool = False):
    """Row `row` of the record `rec` (uint8 [18 d]) from fp64 rows k, v [d]."""
    d = rec.size // 18
    J = d // 32
    for x, c0, s0, is_v in ((k, 0, 16 * d, False), (v, 8 * d, 17 * d, True)):
        code, s = quantise(np.zeros(d) if empty else x)
        bits = scale_bits(s)
        if empty and not is_v:
            bits[:] = 0x8000
        rec[s0 + 2 * row * J:s0 + 2 * (row + 1) * J] = bits.astype("<u2").view(np.uint8)
        for e in range(d):
            j, w = e // 32, e % 32
            if is_v:
                word = ((row // 8) * 32 + (w // 4) * 4 + (row % 8) // 2) * J + j
                nib = (row % 2) * 4 + w % 4
            else:
                word = ((row // 8) * 32 + (row % 8) * 4 + w // 8) * J + j
                nib = w % 8
            at = c0 + 4 * word + nib // 2
            sh = 4 * (nib % 2)
            rec[at] = (int(rec[at]) & ~(15 << sh) & 255) | ((int(code[e]) + 8) << sh)


def write_rows(recs: np.ndarray, rec: np.ndarray, row: np.ndarray, k: np.ndarray, v: np.ndarray, empty=None):
    """write_row for many at once: row[i] of the record recs[rec[i]] (uint8
    [records][18 d], no place twice) from fp64 rows k[i], v[i] [d]."""
    n, d = k.shape
    J = d // 32
    none = np.zeros(n, bool) if empty is None else np.asarray(empty, bool)
    rec, row = np.asarray(rec)[:, None], np.asarray(row)[:, None]
    e = np.arange(0, d, 2)[None]                                  # a byte: elements e and e + 1
    j, w = e // 32, e % 32
    for x, c0, s0, is_v in ((k, 0, 16 * d, False), (v, 8 * d, 17 * d, True)):
        code, s = quantise(np.where(none[:, None], 0.0, x))
        bits = scale_bits(s)
        if not is_v:
            bits[none] = 0x8000
        for i in range(2):
            recs[rec, s0 + 2 * (row * J + np.arange(J)[None]) + i] = (bits >> (8 * i)).astype(np.uint8)
        if is_v:
            word, byte = ((row // 8) * 32 + (w // 4) * 4 + (row % 8) // 2) * J + j, (row % 2) * 2 + w % 4 // 2
        else:
            word, byte = ((row // 8) * 32 + (row % 8) * 4 + w // 8) * J + j, w % 8 // 2
        recs[rec, c0 + 4 * word + byte] = (code[:, 0::2] + 8) | ((code[:, 1::2] + 8) << 4)


def read_row(rec: np.ndarray, row: int):
    """(k, v, empty) of a record's row, fp64."""
    d = rec.size // 18
    J = d // 32
    out = []
    for c0, s0, is_v in ((0, 16 * d, False), (8 * d, 17 * d, True)):
        bits = rec[s0 + 2 * row * J:s0 + 2 * (row + 1) * J].copy().view("<u2").astype(np.uint32)
        s = (bits << 16).view(np.float32).astype(np.float64)
        e = np.arange(d)
        j, w = e // 32, e % 32
        if is_v:
            word, nib = ((row // 8) * 32 + (w // 4) * 4 + (row % 8) // 2) * J + j, (row % 2) * 4 + w % 4
        else:
            word, nib = ((row // 8) * 32 + (row % 8) * 4 + w // 8) * J + j, w % 8
        code = ((rec[c0 + 4 * word + nib // 2].astype(np.int64) >> (4 * (nib % 2))) & 15) - 8
        out.append((code, s))
    empty = bool(np.signbit(out[0][1][0]))
    return out[0][0] * np.repeat(out[0][1], 32), out[1][0] * np.repeat(out[1][1], 32), empty


class Book:
    """table (lists), lens, refs of a paged cache."""

    def __init__(self, n_seqs, n_pages, page_rows, max_pages):
        self.P, self.M, self.n_pages = page_rows, max_pages, n_pages
        self.table = [[-1] * max_pages for _ in range(n_seqs)]
        self.lens = [0] * n_seqs
        self.refs = [0] * n_pages

    def held(self, s):
        return -(-self.lens[s] // self.P)

    def reserve(self, add):
        """pos (or -1) per slot and the copies made [(src, dst, rows)]."""
        wants, pos = [], []
        for s, a in enumerate(add):
            n = self.lens[s]
            if a < 0 or n + a > self.M * self.P:
                wants.append(None)
                continue
            shared = a > 0 and n % self.P != 0 and self.refs[self.table[s][n // self.P]] > 1
            wants.append((shared, -(-(n + a) // self.P) - self.held(s) + shared))
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        copies, dropped, at, out = [], [], 0, False
        for s, w in enumerate(wants):
            if w is None or (w[1] > 0 and (out or at + w[1] > len(free))):
                out = out or w is not None
                pos.append(-1)
                continue
            shared, need = w
            mine = free[at:at + need]
            at += need
            n = self.lens[s]
            pos.append(n)
            if shared:
                old = self.table[s][n // self.P]
                dropped.append(old)
                self.table[s][n // self.P] = mine[0]
                copies.append((old, mine[0], n % self.P))
            for i, p in enumerate(mine[1:] if shared else mine):
                self.table[s][self.held(s) + i] = p
            for p in mine:
                self.refs[p] = 1
            self.lens[s] = n + add[s]
        for p in dropped:
            self.refs[p] -= 1
        return pos, copies

    def fork(self, parent):
        table, lens = [list(t) for t in self.table], list(self.lens)
        for s, p in enumerate(parent):
            if p == s or p < -1 or p >= len(lens):
                continue
            self.table[s] = list(table[p]) if p >= 0 else [-1] * self.M
            self.lens[s] = lens[p] if p >= 0 else 0
        self.refs = [0] * self.n_pages
        for s in range(len(lens)):
            for c in range(self.held(s)):
                self.refs[self.table[s][c]] += 1

    def pack(self):
        """The number of pages in use and the moves [(src, dst)]."""
        n = sum(r > 0 for r in self.refs)
        moves = list(zip([p for p in range(n, self.n_pages) if self.refs[p] > 0],
                         [p for p in range(n) if self.refs[p] == 0]))
        to = dict(moves)
        for a, z in moves:
            self.refs[z], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return n, moves


def attention(q, k, v, empty, scale):
    """fp64 q [G][d] over rows k, v [n][d], empty slots left out: the outputs
    [G][d], and what bounds their rounding: the largest sum |q k| scale, and
    sum_j p_j |v_j|."""
    keep = ~np.asarray(empty, bool)
    k, v = k[keep], v[keep]
    if k.shape[0] == 0:
        z = np.zeros_like(q)
        return z, 0.0, z
    x = scale * (q @ k.T)
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, float((np.abs(q) @ np.abs(k).T).max() * scale), p @ np.abs(v)
