"""The most work that one attention call takes, and what it says of numbers on the device that it cuts or refuses."""

import math

import pytest
import torch

from paged_util import DEV, Batch, attention, check_rows_of, gen, stream_of
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu
LIMIT = 1 << 30


def many_cost(hkv, rows, keys):
    return hkv * -(-rows // 128) * (-(-keys // 64) + 2)


def few_cost(hkv, keys):
    return hkv * (-(-keys // 16) + 6)


def same_everywhere(out, lse, parts, group, scale):
    """Every row of a batch whose rows are all one and the same query over the same keys, against the one row in 64 bits; some of them by check_rows_of."""
    for i in {0, 1, len(out) // 2, len(out) - 1}:
        check_rows_of(out[i:i + 1], lse[i:i + 1], parts, group, scale, i)
    # (the bounds of check_rows_of for this one row, for all of them at once)
    want, want_lse, mass, size, n = attention(parts, group, scale)
    e = size * (want.shape[-1] + 4) * 2.0 ** -23
    rel = 2 * e + 2.0 ** -20 + (n + 64) * 2.0 ** -23
    tol = (2.0 ** -8 * want.abs() + (2.0 ** -8 * (1 + 2.0 ** -7) + 2 * rel)[..., None] * mass).float()
    lse_tol = (e + 2.0 ** -20 + (n + 64) * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()).float()
    for a in range(0, len(out), 1 << 14):
        assert ((out[a:a + (1 << 14)].float() - want.float()).abs() <= tol).all(), a
        assert ((lse[a:a + (1 << 14)] - want_lse.float()).abs() <= lse_tol).all(), a


def test_many_rows_past_2_to_the_26th_tiles():
    """2048 sequences of 128 queries about one prefix: few keys, many rows."""
    n, queries, hkv, group, d, keys = 2048, 128, 8, 8, 64, 32768
    cost = many_cost(hkv, n * queries * group, keys)
    assert 1 << 26 < cost < LIMIT
    g = gen(1)
    table, pools, k, v = stream_of([keys], [0], 1, hkv, d, 64, g)
    own, own_pools, _, _ = stream_of([0], [0], 1, hkv, d, 64, g)
    q = torch.randn(1, hkv * group, d, generator=g).bfloat16().to(DEV)
    rows = q.expand(n * queries, hkv * group, d)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = paged.attend(paged.Stream(rows, *own_pools, own.pages, own.lens), shared=paged.Stream(rows, *pools, table.pages, table.lens),
                            seq_ids=torch.zeros(n, dtype=torch.int32, device=DEV), starts=torch.arange(0, n * queries + 1, queries, dtype=torch.int32, device=DEV),
                            max_queries=queries, status=status)
    assert int(status) == qc.QC_OK
    same_everywhere(out, lse, [(q, k[0], v[0], torch.tensor([keys], device=DEV))], group, 1 / math.sqrt(d))


def test_few_rows_past_2_to_the_26th_tiles():
    """2048 sequences that all are the same row of the table, of 1024 KV heads."""
    n, hkv, d, keys = 2048, 1024, 64, 480
    assert 1 << 26 < n * few_cost(hkv, keys) < LIMIT
    g = gen(2)
    table, pools, k, v = stream_of([keys], [0], 1, hkv, d, 16, g)
    q = torch.randn(1, hkv, d, generator=g).bfloat16().to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = paged.attend(paged.Stream(q.expand(n, hkv, d), *pools, table.pages, table.lens), seq_ids=torch.zeros(n, dtype=torch.int32, device=DEV), status=status)
    assert int(status) == qc.QC_OK
    same_everywhere(out, lse, [(q, k[0], v[0], torch.tensor([keys], device=DEV))], 1, 1 / math.sqrt(d))


@pytest.mark.parametrize("times", [1, 2])
def test_a_batch_of_too_many_tiles_is_refused_and_leaves_everything_as_it_was(times):
    """The same with 8 100 keys: 2^30 and some; of the prefix of a group for each sequence as well, so that the sum itself passes 2^31."""
    n, hkv, d, keys = 2048, 1024, 64, 8128
    assert n * few_cost(hkv, keys) > LIMIT
    table = paged.PageTable.empty(1, keys // 16, 16, keys // 16)
    pool = torch.zeros(keys // 16, hkv, 16, d, dtype=torch.bfloat16, device=DEV)
    paged.table_extend(table, torch.tensor([keys], dtype=torch.int32, device=DEV), max_slots=keys)
    q = torch.zeros(1, hkv, d, dtype=torch.bfloat16, device=DEV).expand(n, hkv, d)
    zeros, own = torch.zeros(n, dtype=torch.int32, device=DEV), paged.Stream(q, pool, pool, table.pages, table.lens)
    out, status = torch.full((n, hkv, d), 3.0, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    shared = dict(shared=own, groups=torch.arange(n + 1, dtype=torch.int32, device=DEV), shared_ids=zeros) if times == 2 else {}
    paged.attend(own, seq_ids=zeros, out=out, status=status, **shared)
    assert int(status) == qc.QC_ERR_PLAN and (out == 3).all()


@pytest.mark.parametrize("group", [1, 40])
@pytest.mark.parametrize("power", [-100, 100, 108])
def test_values_far_from_one(power, group):
    """Values of 600 keys whose sizes add up to some 2^118 at most (5 of them a standard deviation are 2^2.4 each)."""
    b = Batch(5, [300, 7], [1, 1], [(0, 1, 300)], 1, group, 128, 16)
    for pool in (b.pools[1], b.shared[1][1]):
        pool.mul_(2.0 ** power)
    b.values, b.shared = [v * 2.0 ** power for v in b.values], (*b.shared[:3], [v * 2.0 ** power for v in b.shared[3]])
    out, lse = b.call()
    b.check(out, lse)


@pytest.mark.parametrize("power", [11, 13, 16, 57])
@pytest.mark.parametrize("group", [1, 40])
def test_scores_far_from_one(group, power):
    """Products of 2^22 to 2^118 that add up to 2^125 at most: what a key of the largest score weighs is all.

    That weight is 2^x where x is the rounding of the reference, half a step of it or half a doubling below 2^24, so it need not be 1: it is
    rounded to bf16 for its product, 2^-8 of itself, but not for the sum that it is divided by, and the quotient is rounded once more, 2^-8."""
    b = Batch(6, [300, 7], [1, 1], [(0, 1, 300)], 1, group, 128, 16)
    b.q.mul_(2.0 ** power)
    for pool in (b.pools[0], b.shared[1][0]):
        pool.mul_(2.0 ** power)
    out, lse = b.call()
    for i in range(2):
        parts = [(q.double(), k.double() * 2.0 ** power, v, seen) for q, k, v, seen in b.parts(i)]
        best = torch.cat([torch.einsum("qgd,ld->qgl", q, k[:, 0]) for q, k, _, _ in parts], -1)
        top, at = best.max(-1)
        second = best.scatter(-1, at[..., None], -math.inf).amax(-1)
        clear = top - second > 1e-4 * top.abs()      # (else fp32 does not tell them apart)
        values = torch.cat([v[:, 0] for _, _, v, _ in parts])
        want = values[at][clear].double()
        assert clear.float().mean() > 0.9 and ((out[i:i + 1][clear].double() - want).abs() <= want.abs() * (2.0 ** -7 + 2.0 ** -15)).all()
        assert ((lse[i:i + 1].double() / (top * b.scale) - 1).abs() < 1e-4).all()


@pytest.mark.parametrize("group", [1, 40])
@pytest.mark.parametrize("low", [-2.0 ** 28, -2.0 ** 33, -2.0 ** 100])
def test_scores_that_begin_far_below_the_others(group, low):
    """The first keys of each stream score so low that they weigh nothing beside the rest, and sequence 1 has only such keys."""
    b = Batch(7, [200, 70, 300], [1, 1, 2], [(0, 1, 300), (2, 3, 150)], 1, group, 128, 16)
    b.q[:, :, 0] = 1.0
    drop = {0: 130, 1: 70, 2: 65}
    for t, pools, keys, ids, counts in ((b.table, b.pools, b.keys, b.ids, drop), (b.shared[0], b.shared[1], b.shared[2], b.shared_ids, {0: 90, 1: 150})):
        for i, n in counts.items():
            pos = torch.arange(n, device=DEV)
            pools[0][t.pages[int(ids[i])].long()[pos // 16], :, pos % 16, 0] = low / b.scale
    out, lse = b.call()
    # Sequence 1: which of its keys weighs what is lost in the roundings of scores of this size, but its row is a mean of its values.
    row, score = b.begin[1], float(torch.tensor(low / b.scale).bfloat16()) * b.scale
    assert (lse[row].double() / score - 1).abs().max() < 1e-4
    assert (out[row].double() >= b.values[1].double().amin(0) - 0.05).all() and (out[row].double() <= b.values[1].double().amax(0) + 0.05).all()
    # the keys that weigh nothing are left out
    for i in (0, 2):
        n = drop[i]
        b.keys[i], b.values[i] = b.keys[i][n:], b.values[i][n:]
        b.lens[i] -= n
    for i, n in {0: 90, 1: 150}.items():
        b.shared[2][i], b.shared[3][i] = b.shared[2][i][n:], b.shared[3][i][n:]
    b.groups = [(a, z, len(b.shared[2][i])) for i, (a, z, _) in enumerate(b.groups)]
    b.check(out, lse, [0, 2])


@pytest.mark.parametrize("group", [2, 20])
@pytest.mark.parametrize("power", [9, 11, 16])
def test_large_scores_beside_a_value_that_is_not_seen(group, power):
    """The last token's value is infinite; the queries ahead of it do not see it, and all of their elements are of the key that is largest."""
    b = Batch(8, [300, 300], [3, 3], [(0, 1, 300)], 1, group, 128, 16)
    b.q.mul_(2.0 ** power)
    for pool in (b.pools[0], b.shared[1][0]):
        pool.mul_(2.0 ** power)
    for i in range(2):
        b.pools[1][int(b.table.pages[int(b.ids[i]), 299 // 16]), 0, 299 % 16] = math.inf
    out, _ = b.call()
    for i in range(2):
        for j in range(2):      # queries that do not see it
            token = b.begin[i] + j
            best, values = [], []
            for q, k, v, seen in b.parts(i):
                n = int(seen[j])
                best.append(q[j].double() @ k[:n, 0].double().T * 2.0 ** power * b.scale)
                values.append(v[:n, 0].double())
            best, values = torch.cat(best, -1), torch.cat(values)
            top, at = best.max(-1)
            second = best.scatter(-1, at[:, None], -math.inf).amax(-1)
            clear = top - second > torch.maximum(1e-4 * top.abs(), torch.tensor(40.0, device=DEV))
            want = values[at][clear]
            # (a weight's rounding to bf16 and the output's, as for large scores above)
            assert clear.float().mean() > 0.8 and ((out[token][clear].double() - want).abs() <= want.abs() * (2.0 ** -7 + 2.0 ** -15)).all(), (i, j)


def room_of(b):
    return b.table.pages.shape[1] * 16


def test_a_length_beyond_the_table_is_cut_and_said():
    """Every page of the table is there, so that nothing else is to be said."""
    b = Batch(3, [40, 64], [1, 1], [(0, 1, 20)], 1, 2, 64, 16)
    row, room = int(b.ids[1]), room_of(b)
    have = torch.arange(room // 16, device=DEV) % b.pools[0].shape[0]
    b.table.pages[row] = have.to(torch.int32)
    for p in b.pools:
        p.nan_to_num_(0.25)
    b.keys[1], b.values[1] = (p[have].transpose(1, 2).flatten(0, 1) for p in b.pools)
    b.table.lens[row] = room + 1000
    b.lens[1] = room
    out, lse = b.call()
    assert int(b.table.state[1]) == qc.QC_ERR_PLAN
    # (its keys may be sequence 0's pages too: what a page holds is what both see)
    page = b.table.pages[int(b.ids[0])].long()
    pos = torch.arange(40, device=DEV)
    b.keys[0], b.values[0] = (p[page[pos // 16], :, pos % 16] for p in b.pools)
    b.check(out, lse)


def test_a_negative_length_counts_as_none_and_is_said():
    b = Batch(4, [40, 64], [1, 1], [(0, 1, 20)], 1, 2, 64, 16)
    b.table.lens[int(b.ids[0])] = -5
    out, lse = b.call()
    assert int(b.table.state[1]) == qc.QC_ERR_PLAN
    b.keys[0], b.values[0], b.lens[0] = b.keys[0][:0], b.values[0][:0], 0
    b.check(out, lse)
