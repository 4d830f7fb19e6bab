"""Query rows that are computed together (a KV head's group, a sequence's query tokens): a row's result does not depend on what
the rows beside it hold, however large, infinite or no numbers at all."""

import pytest
import torch

from paper_2602_01901_b200 import quant

from quant_util import DEV, check_attend
from test_gpu_quant_attend import Cache, i32, queries

pytestmark = pytest.mark.gpu

# (KV heads, group, query tokens): 2, 4, 8 and 16 rows computed together, in one unit and in several
SHAPES = [(1, 2, [1, 1]), (2, 1, [2, 1]), (1, 4, [1, 1]), (1, 2, [2, 2]), (1, 8, [1, 1]), (2, 3, [3, 1]), (1, 16, [1, 1]), (1, 4, [4, 3]), (1, 5, [16, 2])]


def places(starts, heads):
    return [(t, h) for t in range(starts[-1]) for h in range(heads)]


@pytest.mark.parametrize("head_dim,page", [(64, 32), (128, 16)])
@pytest.mark.parametrize("kv_heads,group,counts", SHAPES, ids=str)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan"), 2.0 ** 101, -(2.0 ** 110), 3.0e38], ids=str)
def test_a_row_that_has_no_scores_leaves_the_others_alone(bad, kv_heads, group, counts, head_dim, page):
    lens, heads = [150, 70], kv_heads * group
    c = Cache(lens, kv_heads, head_dim, page, 3 * head_dim + group)
    starts, q = queries(counts, heads, head_dim, 7 + group)
    at = places(starts, heads)
    victims = at[:: max(2, len(at) // 3)]
    for n, (t, h) in enumerate(victims):
        q[t, h, (17 * n + 3) % head_dim] = bad
    out, lse = quant.attend(c.stream(q.to(DEV)), kv_heads, page, seq_ids=c.ids, starts=i32(starts), max_queries=max(counts))
    for t, h in victims:
        assert torch.isnan(out[t, h].float()).all() and torch.isnan(lse[t, h]), (t, h)
    clean = q.clone()
    for t, h in victims:      # their rows are looked at above; here they are what the oracle says of a row of zeros
        clean[t, h] = 0
    zero, zero_lse = quant.attend(c.stream(clean.to(DEV)), kv_heads, page, seq_ids=c.ids, starts=i32(starts), max_queries=max(counts))
    mixed, mixed_lse = out.clone(), lse.clone()
    for t, h in victims:
        mixed[t, h], mixed_lse[t, h] = zero[t, h], zero_lse[t, h]
    check_attend(mixed, mixed_lse, starts, None, lens, clean, c.k_held, c.v_held, group, head_dim ** -0.5)


@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("kv_heads,group,counts", SHAPES, ids=str)
@pytest.mark.parametrize("spread", [20, 30, 60, 90])
def test_rows_of_very_different_size_have_their_own_accuracy(spread, kv_heads, group, counts, head_dim, page):
    """One row of every few is 2^spread times as large as those beside it."""
    lens, heads = [150, 70], kv_heads * group
    c = Cache(lens, kv_heads, head_dim, page, 5 * head_dim + group)
    starts, q = queries(counts, heads, head_dim, 3 + group)
    for t, h in places(starts, heads)[1::3]:
        q[t, h] = (q[t, h].float() * 2.0 ** spread).bfloat16()
    out, lse = quant.attend(c.stream(q.to(DEV)), kv_heads, page, seq_ids=c.ids, starts=i32(starts), max_queries=max(counts))
    check_attend(out, lse, starts, None, lens, q, c.k_held, c.v_held, group, head_dim ** -0.5)


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (1, 4), (2, 8), (1, 16)])
def test_a_row_gets_the_same_bits_beside_any_other(kv_heads, group):
    """The first head's row alone decides the first head's output: bit for bit the same beside zeros, ordinary and huge rows."""
    lens, heads, head_dim = [700, 33], kv_heads * group, 128
    c = Cache(lens, kv_heads, head_dim, 16, 9)
    starts, q = queries([1, 1], heads, head_dim, 1)
    want = None
    for factor in (1.0, 0.0, 2.0 ** 40, float("inf")):
        x = q.clone()
        x[:, 1:] = 0 if factor == 0 else (x[:, 1:].float() * factor).bfloat16()
        out, lse = quant.attend(c.stream(x.to(DEV)), kv_heads, 16, seq_ids=c.ids)
        if want is None:
            want = out[:, 0].clone(), lse[:, 0].clone()
        assert torch.equal(out[:, 0], want[0]) and torch.equal(lse[:, 0], want[1]), factor
