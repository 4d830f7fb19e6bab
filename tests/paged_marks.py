"""Streams whose outputs count their keys, for attention over bf16 pages: a key that is lost, taken twice or taken from another row shows at
any length, where values of random size drown it.

A key's score is a whole number of doublings e, so that its weight is 2^e, and its value is ``value`` in one channel, which 16 keys in a row
share.  A channel of an output is then the sum of the weights of its keys, over the sum of all: numbers that are known exactly."""

import math
from typing import NamedTuple

import numpy as np

SCALE = math.log(2.0)      # rounds to a factor of 1.0 on the scores in doublings


class Marks(NamedTuple):
    """Of one row of a table: keys, its channels (from `first` on, `channels` of them, the first key's being number `turn`), the value, and the
    doublings of each key's weight."""

    n: int
    turn: int
    first: int
    channels: int
    value: float
    doublings: np.ndarray


def marks(n, turn=0, first=0, channels=128, value=1.0, doublings=0):
    d = np.broadcast_to(np.asarray(doublings), (-(-n // 16),)) if np.ndim(doublings) else np.full(-(-n // 16), doublings)
    return Marks(n, turn, first, channels, value, np.repeat(d, 16)[:n])


def channel_of(m, head, key):
    """(A head's keys begin at a channel of their own.)"""
    return m.first + (key // 16 + 5 * head + m.turn) % m.channels


def counts(parts, head, d):
    """(sum of weights, weighted value of each channel) of keys [(marks, keys seen)]: a number is a list of keys from the first on, an array the keys themselves."""
    total, by = 0.0, np.zeros(d)
    for m, seen in parts:
        keys = np.asarray(seen) if np.ndim(seen) else np.arange(max(0, seen))
        w = np.exp2(m.doublings[keys].astype(np.float64))
        total += w.sum()
        np.add.at(by, channel_of(m, head, keys), w * m.value)
    return total, by


def check_counts(out, lse, total, by, keys, where=""):
    """One output row against its counts.

    Weights are powers of two, so their rounding to bf16 is none.  Where all of them are 1 (exp2 of 0), sums are whole numbers below 2^24 and
    exact.  Else an exponential is off by 2^-22, a lane adds an eighth of the keys one after the other, 2^-24 of the sum each, and
    64 times more between lanes and pieces.  lse is a logarithm (2^-23 of itself), a sum with the reference and a product (2^-24 each).
    An output is a quotient of two such sums, rounded to bf16."""
    even = total == keys
    off = 0.0 if even else 2.0 ** -21 + (keys / 8 + 64) * 2.0 ** -24
    want = by / total
    far = np.abs(out - want) > want * (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * off)
    assert not far.any(), (where, [(int(c), float(out[c] * total), float(by[c])) for c in far.nonzero()[0][:4]])
    assert abs(lse - math.log(total)) <= off + 2.0 ** -22 * max(1.0, abs(math.log(total))) + (0.0 if even else 2.0 ** -19), (where, math.exp(lse), total)
