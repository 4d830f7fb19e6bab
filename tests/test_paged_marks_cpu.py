"""The check of counted keys finds what the tests of long streams are for: mistakes planted in the numbers that it is given (no GPU needed)."""

import math

import numpy as np
import pytest
import torch

from paged_marks import SCALE, check_counts, counts, marks

D = 128


def shown(parts, head=0):
    """What a kernel without a mistake gives: (out, lse)."""
    total, by = counts(parts, head, D)
    return torch.tensor(by / total).bfloat16().double().numpy(), float(np.float32(math.log(total)))


def found(given, parts, head=0):
    total, by = counts(parts, head, D)
    keys = sum(seen for _, seen in parts)
    check_counts(*shown(parts, head), total, by, keys)
    with pytest.raises(AssertionError):
        check_counts(*shown(given, head), total, by, keys)


def test_the_scale_is_one_doubling():
    assert np.float32(SCALE) * np.float32(1.4426950408889634) == np.float32(1.0)


LONG = [(marks(30017), 30017), (marks(20011, value=3.0), 20011)]


@pytest.mark.parametrize("keys", [[0], [20010], [12345], range(64, 128), range(10000, 10016), range(9000, 9256)])
def test_lost_and_doubled_keys_of_a_long_stream(keys):
    every, keys = np.arange(20011), np.array(list(keys))
    found([LONG[0], (LONG[1][0], np.delete(every, keys))], LONG)
    found([LONG[0], (LONG[1][0], np.concatenate([every, keys]))], LONG)
    found([(LONG[0][0], np.delete(np.arange(30017), keys)), LONG[1]], LONG)


@pytest.mark.parametrize("n,instead", [(16, 16 * 7), (16, 16), (64, 64 * 9)])
def test_keys_of_another_place_or_another_head(n, instead):
    every = np.arange(20011)
    moved = every.copy()
    moved[8000:8000 + n] += instead
    found([LONG[0], (LONG[1][0], moved)], LONG)
    total, by = counts(LONG, 0, D)
    with pytest.raises(AssertionError):
        check_counts(*shown(LONG, 1), total, by, 50028)


@pytest.mark.parametrize("key", [0, 500, 1023])
def test_one_key_of_any_weight_where_each_tile_has_a_channel(key):
    rng = np.random.default_rng(key)
    parts = [(marks(1024, 0, 0, 64, 1.0, rng.integers(-12, 13, 64)), 1024), (marks(1000, 0, 64, 64, 1.0, rng.integers(-12, 13, 63)), 1000)]
    found([(parts[0][0], np.delete(np.arange(1024), [key])), parts[1]], parts)
    found([parts[0], (parts[1][0], np.append(np.arange(1000), min(key, 999)))], parts)
