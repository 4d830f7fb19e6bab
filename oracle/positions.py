"""CPU oracle of norms and rotations of query and key rows, in numpy and 64 bits.

Written from the definitions, element by element of a row; shares nothing with the library.  Test infrastructure only.
"""

from __future__ import annotations

import math

import numpy as np


def pair_of(e: int, pairs: int, adjacent: bool):
    """(pair, whether e is its second element, the other element) of element e of a row; None where it does not turn."""
    if e >= 2 * pairs:
        return None
    if adjacent:
        return e // 2, e % 2 == 1, e ^ 1
    return e % pairs, e >= pairs, (e + pairs) % (2 * pairs)


def normed(x, weight, eps: float) -> np.ndarray:
    """x [..., d] / sqrt(mean x^2 + eps) * weight; x itself where weight is None."""
    x = np.asarray(x, np.float64)
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)


def turned(x, positions, freqs, axes, adjacent: bool) -> np.ndarray:
    """x [tokens, heads, d], positions [axes, tokens]: every pair turned by its angle."""
    x, out = np.asarray(x, np.float64), np.array(x, np.float64)
    pairs = len(freqs)
    for e in range(x.shape[-1]):
        found = pair_of(e, pairs, adjacent)
        if found is None:
            continue
        pair, second, other = found
        for t in range(x.shape[0]):
            angle = math.remainder(int(positions[axes[pair]][t]) * float(freqs[pair]), 2 * math.pi)
            out[t, :, e] = x[t, :, e] * math.cos(angle) + (1 if second else -1) * x[t, :, other] * math.sin(angle)
    return out
