"""CPU oracle of a K/V cache in 4 bits, in numpy and 64 bits: rows, page tables, attention.

Written from the definitions (the format of a page as `include/qc.h` states it, softmax attention), one row or one
token at a time; shares nothing with the library.  Test infrastructure only.
"""

from __future__ import annotations

import math

import numpy as np


def bf16(x: float) -> float:
    """Nearest bf16 value, ties to even, of a finite number in the normal range."""
    if x == 0:
        return 0.0
    m, e = math.frexp(x)                      # x = m * 2^e, 1/2 <= |m| < 1
    scaled = m * 256.0                        # 8 bits in front of the point
    down = math.floor(scaled)
    rest = scaled - down
    if rest > 0.5 or (rest == 0.5 and down % 2 == 1):
        down += 1
    return math.ldexp(down, e - 8)


def quantise(row) -> tuple[float, float, np.ndarray]:
    """(lo, r, codes) of one row of bf16 values."""
    row = np.asarray(row, np.float64)
    lo, hi = float(row.min()), float(row.max())
    span = hi - lo
    if not np.isfinite(row).all() or span > 3.4028234663852886e38:
        return math.nan, 0.0, np.zeros(len(row), np.int64)
    if span < 2.0 ** -100:
        return lo, 0.0, np.zeros(len(row), np.int64)
    r = bf16(15.0 / span)
    return lo, r, np.rint((row - lo) * r).astype(np.int64)


def value(lo: float, r: float, codes) -> np.ndarray:
    codes = np.asarray(codes, np.float64)
    return lo + (codes / r if r else 0.0 * codes)


# ---- where things lie in a page -----------------------------------------------------------------

def page_bytes(heads: int, head_dim: int, page: int) -> int:
    return heads * page * (head_dim // 2 + 4)


def code_place(which: str, head_dim: int, head: int, page: int, token: int, d: int) -> tuple[int, int]:
    """(byte inside the page, 0 for its low and 1 for its high half) of element d of a token's row."""
    block, i = divmod(token, 16)
    base = (head * (page // 16) + block) * 8 * head_dim
    if which == "k" and head_dim == 128:
        at = np.ravel_multi_index((i % 2, i // 2, d // 32, d // 2 % 16), (2, 8, 4, 16))
    elif which == "k":
        at = np.ravel_multi_index((i // 2, d // 16, i % 2, d // 2 % 8), (8, 4, 2, 8))
    elif head_dim == 128:
        at = np.ravel_multi_index((d // 8 % 2, d // 16, i // 4, d // 2 % 4, i % 4), (2, 8, 4, 4, 4))
    else:
        at = np.ravel_multi_index((d // 8, i // 4, d // 2 % 4, i % 4), (8, 4, 4, 4))
    return base + int(at), d % 2


def row_at(pool: np.ndarray, which: str, heads: int, head_dim: int, page: int, slot: int, head: int):
    """(lo, r, codes) of the row that a pool's bytes [pages, page bytes] hold at a slot."""
    raw = pool[slot // page]
    token = slot % page
    codes = np.empty(head_dim, np.int64)
    for d in range(head_dim):
        byte, half = code_place(which, head_dim, head, page, token, d)
        codes[d] = (int(raw[byte]) >> (4 * half)) & 15
    at = heads * page * head_dim // 2 + (head * page + token) * 4
    word = raw[at:at + 4].view(np.uint32)[0]
    as_float = lambda bits: float(np.array([bits], np.uint32).view(np.float32)[0])
    return as_float((word & 0xFFFF) << 16), as_float(word & 0xFFFF0000), codes


# ---- page tables -----------------------------------------------------------------------------------

class Refused(Exception):
    pass


class Table:
    """Integer model: lengths, page lists and the free pages as a stack."""

    def __init__(self, max_seqs: int, max_pages: int, page: int, n_pages: int):
        self.page, self.max_pages, self.n_pages = page, max_pages, n_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs

    def _check(self, ids, counts):
        if any(not 0 <= i < len(self.lens) for i in ids) or any(c < 0 for c in counts):
            raise Refused("argument")
        if len(set(ids)) < len(ids):
            raise Refused("state")

    def extend(self, ids, new, max_slots: int):
        self._check(ids, new)
        need = [-(-(self.lens[i] + n) // self.page) - len(self.pages[i]) for i, n in zip(ids, new)]
        if any(len(self.pages[i]) + k > self.max_pages for i, k in zip(ids, need)) or sum(need) > len(self.free):
            raise Refused("pages")
        if sum(new) > max_slots:
            raise Refused("argument")
        starts, slots = [0], []
        for i, n, k in zip(ids, new, need):
            self.pages[i] += [self.free.pop() for _ in range(k)]
            slots += [self.pages[i][t // self.page] * self.page + t % self.page for t in range(self.lens[i], self.lens[i] + n)]
            self.lens[i] += n
            starts.append(len(slots))
        return starts, slots + [-1] * (max_slots - len(slots))

    def trim(self, ids, keep):
        self._check(ids, keep)
        given = []
        for i, n in zip(ids, keep):
            self.lens[i] = min(self.lens[i], n)
            stay = -(-self.lens[i] // self.page)
            given += self.pages[i][stay:]
            del self.pages[i][stay:]
        self.free += given[::-1]


# ---- attention ---------------------------------------------------------------------------------------

def attention(q, streams, scale: float):
    """One query head's row over streams [(query, keys [n, d], values [n, d])] with one softmax: (out, lse)."""
    logits = [np.asarray(k, np.float64) @ np.asarray(s, np.float64) * scale for s, k, _ in streams]
    values = [np.asarray(v, np.float64) for _, _, v in streams]
    logit, val = np.concatenate(logits), np.concatenate(values)
    if logit.size == 0:
        return np.zeros(len(q)), -math.inf
    top = logit.max()
    weight = np.exp(logit - top)
    return (weight / weight.sum()) @ val, top + math.log(weight.sum())
