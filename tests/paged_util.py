"""Seeded rows, positions and rotations for the tests of rows and bf16 pages, with the oracle's view and how far an output may be off."""

import numpy as np
import torch

from oracle import positions as O
from paper_2602_01901_b200 import paged

DEV = "cuda"


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows(n, heads, head_dim, g):
    """bf16 rows on the CPU: channels and tokens of different size."""
    channel = torch.exp(0.5 * torch.randn(heads, head_dim, generator=g))
    token = torch.exp(0.4 * torch.randn(n, 1, 1, generator=g))
    return (torch.randn(n, heads, head_dim, generator=g) * channel * token).bfloat16()


def rotation(rotary, n_axes, g, adjacent=False, theta=10000.0):
    """(Rotation on the device, frequencies, axes) of `rotary` elements; axes in no order."""
    pairs = rotary // 2
    freqs = (theta ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    axes = torch.randint(0, n_axes, (pairs,), generator=g, dtype=torch.int32)
    return paged.Rotation(freqs.to(DEV), axes.to(DEV) if n_axes > 1 else None, adjacent), freqs.tolist(), axes.tolist() if n_axes > 1 else [0] * pairs


def check_rows(got, x, positions, freqs, axes, adjacent, weight, eps):
    """Rows against the oracle.  x [n, heads, d] bf16 on the CPU, positions [axes, n] integers, freqs empty: no rotation.

    With a norm an element is x * scale * w: the sum of d squares is off by (d + 1) 2^-24 of itself at most, the mean and eps add
    2^-23, the reciprocal root halves that and adds 2^-22, and two products 2^-24 each.  An angle is cut off at 2^-32 turns and
    rounded to 2^-24 half turns at most; its sine and cosine are off by 2^-23 more: 2^-21 of the pair's elements together.  Two products and a
    sum round three times, 2^-24 each of |a| + |b|.  Then half a step of bf16, 2^-8."""
    x, got = x.double().numpy(), got.double().cpu().numpy()
    d = x.shape[-1]
    a = O.normed(x, weight, eps)
    want = O.turned(a, positions, freqs, axes, adjacent) if len(freqs) else a
    size = np.abs(a)
    for e in range(2 * len(freqs)):
        size[..., e] = np.abs(a[..., e]) + np.abs(a[..., O.pair_of(e, len(freqs), adjacent)[2]])
    rel = (2.0 ** -21 + 3 * 2.0 ** -24 if len(freqs) else 0.0) + ((d + 3) * 2.0 ** -25 + 2.0 ** -22 + 2.0 ** -23 if weight is not None else 0.0)
    tol = 2.0 ** -8 * np.abs(want) + 2 * rel * size + 2.0 ** -133
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all() and (np.where(fine, 0, got) == np.where(fine, 0, want))[~np.isnan(want)].all()
    far = np.where(fine, np.abs(got - want) / tol, 0)
    assert far.max(initial=0.0) <= 1, (np.unravel_index(far.argmax(), far.shape), far.max())
