"""Angles of far positions: sines and cosines of rotate against the angle in whole numbers of many bits."""

import math

import numpy as np
import pytest
import torch

from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu

BITS = 256


def two_pi():
    """2 pi * 2^BITS, by Machin's formula in whole numbers."""
    def arctan(x):
        term = total = (1 << BITS + 32) // x
        n, sign = 3, -1
        while term:
            term //= x * x
            total, sign, n = total + sign * (term // n), -sign, n + 2
        return total
    return 8 * (4 * arctan(5) - arctan(239)) >> 32


TWO_PI = two_pi()


def turns(freq, position):
    """position * freq / 2 pi, less the nearest whole number: freq is fp32, so a whole number over 2^149."""
    whole = int(np.ldexp(np.float64(np.float32(freq)), 149)) * position
    full = TWO_PI
    whole <<= BITS - 149
    rest = whole % full
    if 2 * rest > full:
        rest -= full
    return (rest << 64) // full * 2.0 ** -64


def near_the_axis(freq, top):
    """Positions of a stretch below `top` whose angle is next to a multiple of a quarter turn: a sine or a cosine there shows the angle's error."""
    step, at = turns(freq, 1), turns(freq, top - 20000)
    quarter = (4 * (at + step * np.arange(20000)) + 0.5) % 1 - 0.5      # (drifts by 20000 * 2^-53 turns)
    return [top - 20000 + int(i) for i in np.argsort(np.abs(quarter))[:6]]


def test_the_oracle_of_this_file():
    assert abs(TWO_PI / 2 ** BITS - 2 * math.pi) < 1e-15
    for freq, position in ((1.0, 1), (0.75, -3), (123.25, 1000), (1e-4, 5)):
        want = math.remainder(float(np.float32(freq)) * position, 2 * math.pi) / (2 * math.pi)
        assert abs(turns(freq, position) - want) < 1e-12


@pytest.mark.parametrize("top", [2 ** 18, 2 ** 24, 2 ** 27, 2 ** 31, -2 ** 31 + 20000])
@pytest.mark.parametrize("freqs", [[1.0, 0.75, 0.1234, 1e-3, 1e-5, -0.5, 0.9999, 2e-7], [123.25, 100.0, 31.7, 6.2831855, -77.7, 3.1415927, 1000.5, 50000.0]])
def test_angles_are_exact_to_a_rounding_of_fp32_at_every_position(freqs, top):
    """Pairs (1, 0) turn into (cos, sin).  The angle is a fraction of 64 bits: off by 2^-63 turns times the position, cut off at 2^-32, and
    rounded to 24 bits of at most one half turn (2^-26 turns): 2 pi (2^-26 + 2^-31) in all.  sincospif adds 2^-22 of the value, the output is rounded to bf16."""
    positions = [p for f in freqs for p in near_the_axis(f, top)]
    x = torch.zeros(len(positions), 1, 64, dtype=torch.bfloat16, device="cuda")
    x[:, :, :8] = 1
    rot = paged.Rotation(torch.tensor(freqs, device="cuda"))
    got, _ = paged.rotate(x, None, torch.tensor(positions, dtype=torch.int32, device="cuda"), rot)
    got = got.double().cpu().numpy()[:, 0]
    angle = np.array([[2 * math.pi * turns(f, p) for f in freqs] for p in positions])
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    assert (np.abs(want) < 1e-3).any(), "no angle that would show its error"
    tol = 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -13) + 2 * math.pi * (2.0 ** -26 + 2.0 ** -31)
    far = np.abs(got[:, :16] - want) / tol
    assert far.max() <= 1, (far.max(), np.unravel_index(far.argmax(), far.shape))
