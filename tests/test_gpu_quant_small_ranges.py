"""Attention over rows whose ranges are near the least that has steps (2^-100; a row below it stands for its smallest element), alone
and among ordinary ones."""

import pytest
import torch

from paper_2602_01901_b200 import quant

from quant_util import DEV, check_attend, gen, held
from test_gpu_quant_attend import Cache, i32, queries

pytestmark = pytest.mark.gpu


def rows_of_range(n, heads, head_dim, low, high, seed):
    """bf16 rows from -x to 2 x, say, their ranges spread over 2^low to 2^high."""
    g = gen(seed)
    x = torch.rand(n, heads, head_dim, generator=g) - 0.3
    x[..., 0], x[..., 1] = 0.0, 1.0
    x = x / (x.max(-1, keepdim=True).values - x.min(-1, keepdim=True).values)
    return (x * 2.0 ** (low + (high - low) * torch.rand(n, heads, 1, generator=g))).bfloat16()


def store(c, i, which, x):
    slot = c.table.pages[int(c.ids[i])].long()[torch.arange(len(x), device=DEV) // c.page] * c.page + torch.arange(len(x), device=DEV) % c.page
    given = [x.to(DEV) if which == n else None for n in "kv"]
    quant.append(*[p if which == n else None for n, p in zip("kv", c.pools)], slot.to(torch.int32), *given, c.page)
    return held(x)


@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 32)])
@pytest.mark.parametrize("group", [1, 3, 8, 16])
@pytest.mark.parametrize("low,high", [(-100, -97), (-99.9, -99.9), (-104, -98)])
def test_values_of_the_least_ranges(low, high, group, head_dim, page):
    lens = [210, 64]
    c = Cache(lens, 1, head_dim, page, 3 + group)
    values = [store(c, i, "v", rows_of_range(n, 1, head_dim, low, high, i + group)) for i, n in enumerate(lens)]
    assert any((v["step"] > 0).any() for v in values) or low == -104
    starts, q = queries([1, 1], group, head_dim, 5)
    out, lse = quant.attend(c.stream(q.to(DEV)), 1, page, seq_ids=c.ids)
    assert (out != 0).any()
    check_attend(out, lse, starts, None, lens, q, c.k_held, values, group, head_dim ** -0.5)


def test_values_of_the_least_ranges_before_and_behind_ordinary_ones():
    """Weights are put on a larger step as one comes by, 2^100 times the first at once."""
    lens = [256, 256]
    c = Cache(lens, 1, 64, 16, 9)
    values = []
    for i, n in enumerate(lens):
        x = rows_of_range(n, 1, 64, -100, -97, i)
        at = slice(128, 256) if i == 0 else slice(0, 128)
        x[at] = c.v[i][at]
        values.append(store(c, i, "v", x))
    starts, q = queries([1, 1], 4, 64, 5)
    out, lse = quant.attend(c.stream(q.to(DEV)), 1, 16, seq_ids=c.ids)
    check_attend(out, lse, starts, None, lens, q, c.k_held, values, 4, 64 ** -0.5)


@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 32)])
def test_keys_of_the_least_ranges(head_dim, page):
    lens, group = [210, 64], 4
    c = Cache(lens, 1, head_dim, page, 3)
    keys = [store(c, i, "k", rows_of_range(n, 1, head_dim, -100, -97, i)) for i, n in enumerate(lens)]
    starts, q = queries([1, 1], group, head_dim, 5, size=2.0 ** 60)
    out, lse = quant.attend(c.stream(q.to(DEV)), 1, page, seq_ids=c.ids, scale=2.0 ** 38)
    check_attend(out, lse, starts, None, lens, q, keys, c.v_held, group, 2.0 ** 38)
