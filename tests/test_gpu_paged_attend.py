"""Attention over bf16 pages, with and without shared prefixes, against softmax attention in 64 bits."""

import math
import random

import pytest
import torch

from paged_util import DEV, Batch, attention, check_rows_of, gen, rotation, rows
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu


def run(b, **change):
    out, lse = b.call(**change)
    assert int(b.table.state[1]) == qc.QC_OK
    b.check(out, lse)
    return out, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193]


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_own_lengths_at_the_edges_of_pages_and_tiles(page, d):
    run(Batch(1, EDGES, [1] * len(EDGES), [], 2, 3, d, page))


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_prefixes_at_the_edges_of_pages_and_tiles(page, d):
    n = len(EDGES)
    run(Batch(2, [i % 5 for i in range(2 * n + 3)], [1] * (2 * n + 3), [(1 + 2 * i, 3 + 2 * i, p) for i, p in enumerate(EDGES)], 2, 2, d, page))


@pytest.mark.parametrize("members,group,queries", [(1, 1, 1), (3, 1, 1), (8, 4, 1), (32, 1, 1), (33, 1, 1), (16, 4, 1), (65, 1, 1), (18, 7, 1), (128, 1, 1), (129, 1, 1), (37, 7, 1), (11, 5, 5),
                                                   (3, 40, 3), (2, 8, 16), (1, 1, 128), (2, 9, 100), (1, 128, 1), (1, 130, 2)])
def test_every_number_of_query_rows(members, group, queries):
    rng = random.Random(members * group)
    lens = [rng.randint(0, 200) for _ in range(members)]
    run(Batch(3, lens, [queries] * members, [(0, members, 150)], 2, group, 128, 16, lazy=True))


@pytest.mark.parametrize("seed", range(12))
def test_batches_of_many_kinds(seed):
    rng = random.Random(seed)
    n = rng.choice([1, 2, 5, 20, 60])
    high, pre = rng.choice([3, 70, 500, 2500]), rng.choice([1, 60, 700, 3000])
    lens = [rng.randint(0, high) for _ in range(n)]
    queries = [rng.randint(0 if n > 1 else 1, rng.choice([1, 3, 9])) for _ in range(n)]
    if sum(queries) == 0:
        queries[0] = 1
    cuts = sorted(rng.randint(0, n) for _ in range(rng.choice([0, 2, 3, 5])))       # (groups may be empty)
    groups = [(a, b, rng.randint(0, pre)) for a, b in zip(cuts, cuts[1:])]
    hkv, group = rng.choice([(1, 1), (4, 7), (8, 4), (2, 16), (32, 1), (3, 5)])
    run(Batch(seed, lens, queries, groups, hkv, group, rng.choice([64, 128]), rng.choice([16, 32, 64]), lazy=rng.random() < 0.5, causal=rng.random() < 0.7,
              scale=rng.choice([0.0, 0.03, 0.2])))


def test_long_streams_are_cut_and_joined():
    b = Batch(5, [9000, 20011, 1], [1, 3, 2], [(0, 2, 30017)], 1, 4, 128, 64)
    first = run(b)
    again = b.call()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])       # the same bits each time


def test_a_large_batch_of_short_sequences():
    rng = random.Random(6)
    n = qc.QC_PAGED_MAX_SEQS
    b = Batch(6, [rng.randint(0, 40) for _ in range(n)], [1] * n, [(5, 900, 70), (900, 900, 3), (900, 2000, 1), (2000, 2048, 333)], 2, 2, 64, 16)
    out, lse = b.call()
    assert int(b.table.state[1]) == qc.QC_OK
    b.check(out, lse, range(0, n, 37))
    b.check(out, lse, [0, 4, 5, 899, 900, 1999, 2000, 2047])


@pytest.mark.parametrize("lens,prefix", [([0] * 19 + [5], 40000), ([0] * 19 + [70], 19000), ([9000] * 20, 1), ([20000] + [0] * 19, 65)])
def test_little_of_one_kind_beside_much_of_the_other(lens, prefix):
    """Rows that single warps take, and rows that a block takes, share the device out between them: neither gets nothing."""
    run(Batch(18, lens, [1] * 20, [(0, 20, prefix)], 1, 1, 128, 64, lazy=True))


@pytest.mark.parametrize("group", [1, 2, 5])
def test_sequences_of_as_many_rows_as_a_warp_takes_and_more(group):
    queries = [3, 8, 16, 9, 17, 1, 4, 33]
    run(Batch(19, [700, 5, 90, 1300, 33, 2000, 64, 400], queries, [(1, 4, 130), (4, 6, 500)], 2, group, 64, 32))


def test_many_groups_of_one():
    n = 300
    run(Batch(7, [3] * n, [1] * n, [(i, i + 1, i % 130) for i in range(n)], 1, 3, 128, 16, lazy=True))


def test_as_many_groups_as_sequences():
    n = qc.QC_PAGED_MAX_SEQS
    b = Batch(33, [i % 7 for i in range(n)], [1] * n, [(i, i + 1, i % 23) for i in range(n)], 1, 2, 64, 16)
    out, lse = b.call()
    assert int(b.table.state[1]) == qc.QC_OK
    b.check(out, lse, list(range(0, n, 61)) + [n - 1])


@pytest.mark.parametrize("hkv,group", [(1024, 1), (1, 1024), (64, 16)])
def test_the_most_heads(hkv, group):
    run(Batch(34, [70, 3, 0], [1, 2, 1], [(0, 2, 90)], hkv, group, 64, 16))


def test_the_most_queries():
    n = qc.QC_PAGED_MAX_QUERIES
    run(Batch(35, [n, 500, 40, 200], [n, n, 33, n - 1], [(1, 4, 300)], 2, 6, 128, 32))


def test_a_prefix_is_the_same_as_rows_of_ones_own():
    """With the same queries for both streams, a prefix of a group and a copy of it ahead of each sequence's own rows give the same, but for roundings."""
    n, p, own, d, hkv, group = 6, 333, [1, 20, 64, 100, 131, 7], 128, 2, 4
    a = Batch(8, own, [1] * n, [(0, n, p)], hkv, group, d, 16)
    out, lse = run(a)
    b = Batch(9, [p + x for x in own], [1] * n, [], hkv, group, d, 16)
    b.q = b.q_shared = a.q
    for i in range(n):
        b.keys[i], b.values[i] = torch.cat([a.shared[2][0], a.keys[i]]), torch.cat([a.shared[3][0], a.values[i]])
        page_ids = b.table.pages[b.ids[i].long()].long()
        pos = torch.arange(p + own[i], device=DEV)
        for pool, x in zip(b.pools, (b.keys[i], b.values[i])):
            pool[page_ids[pos // 16], :, pos % 16] = x
    out2, lse2 = run(b)
    assert (lse - lse2).abs().max() < 1e-5


def test_without_lists_sequences_are_rows_in_order_and_share_one_prefix():
    b = Batch(10, [5, 0, 77], [1, 1, 1], [(0, 3, 200)], 2, 2, 64, 16)
    t, p = b.table, b.shared[0]
    order = b.ids.long()
    want, want_lse = run(b)
    own = paged.Stream(b.q, *b.pools, t.pages[order].contiguous(), t.lens[order].contiguous())
    row = b.shared_ids.long()
    shared = paged.Stream(b.q, *b.shared[1], p.pages[row].contiguous(), p.lens[row].contiguous())
    out, lse = paged.attend(own, shared=shared)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_queries_inside_a_fused_projection_and_one_for_all():
    b = Batch(11, [40, 3, 90], [2, 1, 2], [(0, 2, 70)], 2, 3, 128, 16, lazy=True)
    want = run(b)
    fused = torch.randn(5, 16, 128, device=DEV).bfloat16()
    fused[:, 2:8], fused[:, 9:15] = b.q, b.q_shared
    s = b.shared_stream()
    out = b.call(own=b.stream()._replace(q=fused[:, 2:8]), shared=s._replace(q=fused[:, 9:15]))
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    b.q = b.q[:1].expand(5, 6, 128)
    run(b)


def test_tokens_of_no_sequence_stay_what_they_were():
    b = Batch(12, [4, 30], [1, 2], [(0, 2, 9)], 2, 2, 64, 16)
    padded = lambda q: torch.cat([torch.full((2, 4, 64), math.nan, device=DEV).bfloat16(), q, torch.full((3, 4, 64), math.nan, device=DEV).bfloat16()])
    want, want_lse = run(b)
    out = torch.full((8, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got, lse = b.call(own=b.stream()._replace(q=padded(b.q)), shared=b.shared_stream()._replace(q=padded(b.q)), starts=b.starts + 2, out=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(out[2:5], want) and torch.equal(lse[2:5], want_lse) and (out[:2] == 7).all() and (out[5:] == 7).all()


def test_values_and_queries_that_are_no_numbers_stay_in_their_rows():
    """An infinite value, or a query with a NaN, changes the rows that see it and no other; a key whose score is minus infinity weighs nothing."""
    b = Batch(13, [70, 80, 90, 5], [1, 1, 1, 1], [(0, 2, 100), (2, 3, 40)], 2, 2, 128, 16)
    want, want_lse = run(b)
    at = lambda t, i, pos: (int(t.pages[i, pos // 16]), pos % 16)
    page, place = at(b.table, int(b.ids[1]), 66)
    b.pools[1][page, 0, place, 5] = math.inf                     # sequence 1, first KV head
    page, place = at(b.shared[0], int(b.shared_ids[1]), 39)
    b.shared[1][1][page, 1, place] = math.nan                    # sequence 2, second KV head
    b.q[3, 0, 0] = math.nan                                      # sequence 3, head 0
    out, lse = b.call()
    touched = torch.zeros_like(out, dtype=torch.bool)
    touched[1, :2, 5], touched[2, 2:], touched[3, 0] = True, True, True
    assert torch.equal(out[~touched], want[~touched]) and not out[touched].isfinite().any() and (out[1, :2, 5] == math.inf).all()
    assert lse[3, 0].isnan() and torch.equal(lse[:3], want_lse[:3]) and torch.equal(lse[3, 1:], want_lse[3, 1:])


@pytest.mark.parametrize("group", [2, 10])
def test_what_a_query_does_not_see_may_be_no_number(group):
    """The last own token's value is infinite in one element of one head, its key a NaN in another: queries ahead of it see neither."""
    b = Batch(28, [70, 200], [3, 3], [(0, 2, 100)], 2, group, 128, 16)
    want, want_lse = run(b)
    page, place = int(b.table.pages[int(b.ids[1]), 199 // 16]), 199 % 16
    b.pools[1][page, 0, place, 5] = math.inf
    b.pools[0][page, 1, place, 9] = math.nan
    out, lse = b.call()
    assert (out[5, :group, 5] == math.inf).all() and out[5, group:].isnan().all() and lse[5, group:].isnan().all()
    out[5, :group, 5], out[5, group:], lse[5, group:] = want[5, :group, 5], want[5, group:], want_lse[5, group:]
    b.check(out, lse)


def test_scores_of_minus_infinity():
    b = Batch(14, [64, 130, 65], [1, 1, 1], [(1, 3, 64)], 1, 2, 64, 16)
    b.q[:, :, 0] = 1.0
    row = lambda i: b.table.pages[int(b.ids[i])].long()
    b.pools[0][row(0)[:4], :, :, 0] = -math.inf                  # all keys of sequence 0
    b.pools[0][row(1)[:4], :, :, 0] = -math.inf                  # the first tile of sequence 1
    b.pools[0][row(2)[4], :, 0, 0] = -math.inf                   # the last key of sequence 2
    for i, keep in ((1, slice(64, 130)), (2, slice(0, 64))):
        b.keys[i], b.values[i], b.lens[i] = b.keys[i][keep], b.values[i][keep], 66 if i == 1 else 64
    out, lse = b.call()
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    b.causal = False
    b.check(out, lse, [1, 2])


@pytest.mark.parametrize("spread", [0.01, 1.0, 12.0])
def test_flat_and_peaked_weights(spread):
    run(Batch(15, [300, 10, 0, 1000], [1, 2, 1, 1], [(0, 3, 400)], 2, 4, 128, 16, spread=spread))


def test_scores_that_rise_along_the_keys():
    """The running maximum moves in every tile."""
    b = Batch(16, [700, 400], [1, 1], [(0, 2, 500)], 1, 4, 64, 16)
    for t, pools, keys, ids in ((b.table, b.pools, b.keys, b.ids), (b.shared[0], b.shared[1], b.shared[2], b.shared_ids)):
        for i, k in enumerate(keys):
            k[:, :, 0] = (torch.arange(len(k), device=DEV) * 0.5)[:, None].bfloat16()
            pos = torch.arange(len(k), device=DEV)
            pools[0][t.pages[int(ids[i])].long()[pos // 16], :, pos % 16] = k
    b.q[:, :, 0] = 3.0
    run(b)
    b.q[:, :, 0] = -3.0
    run(b)


def test_a_pool_past_32_bits_of_elements():
    b = Batch(17, [100, 40], [1, 1], [(0, 2, 50)], 32, 1, 128, 16)
    pools = [torch.empty(33000, 32, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    assert pools[0].numel() > 2 ** 31
    move = 33000 - b.pools[0].shape[0]
    for new, old in zip(pools, b.pools):
        new[move:] = old
    want = run(b)
    pages = torch.where(b.table.pages >= 0, b.table.pages + move, -1)
    out, lse = b.call(own=paged.Stream(b.q, *pools, pages, b.table.lens))
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_a_pool_past_32_bits_of_elements_and_many_rows():
    b = Batch(29, [100, 40], [1, 1], [(0, 2, 150)], 32, 20, 128, 16)
    pools = [torch.empty(33000, 32, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    move = 33000 - b.shared[1][0].shape[0]
    for new, old in zip(pools, b.shared[1]):
        new[move:] = old
    want = run(b)
    s = b.shared_stream()
    out, lse = b.call(shared=s._replace(k_pool=pools[0], v_pool=pools[1], pages=torch.where(s.pages >= 0, s.pages + move, -1)))
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_the_same_row_more_than_once():
    b = Batch(30, [50, 40, 90, 20], [1, 2, 1, 1], [(0, 1, 70), (1, 3, 70), (3, 4, 300)], 2, 4, 64, 16)
    run(b)
    ids, shared_ids = b.ids[torch.tensor([0, 2, 2, 0], device=DEV)], b.shared_ids[torch.tensor([0, 0, 2], device=DEV)]
    b.keys, b.values = [[x[i] for i in (0, 2, 2, 0)] for x in (b.keys, b.values)]
    b.lens = [50, 90, 90, 50]
    b.shared = (b.shared[0], b.shared[1], *[[x[i] for i in (0, 0, 2)] for x in b.shared[2:]])
    out, lse = b.call(seq_ids=ids, shared_ids=shared_ids)
    b.check(out, lse)


# ---- numbers on the device that do not fit ---------------------------------------------------------------------------

@pytest.mark.parametrize("name,at,value", [
    ("starts", 0, -1), ("starts", 1, 7), ("starts", 3, 9), ("starts", 2, 0), ("seq_ids", 1, 5), ("seq_ids", 0, -1), ("groups", 0, -1), ("groups", 1, 4), ("groups", 1, -2), ("groups", 2, 5),
    ("shared_ids", 0, 3), ("shared_ids", 1, -1),
])
def test_lists_that_do_not_fit_leave_everything_as_it_was(name, at, value):
    b = Batch(18, [5, 60, 7], [1, 2, 1], [(0, 2, 9), (2, 3, 70)], 2, 2, 64, 16)
    lists = dict(starts=b.starts, seq_ids=b.ids, groups=b.group_starts, shared_ids=b.shared_ids)
    bad = lists[name].clone()
    bad[at] = value
    out = torch.full_like(b.q, 3.0)
    b.call(**{name: bad}, out=out)
    assert (out == 3).all()
    with pytest.raises(qc.QcError) as e:
        b.table.check()
    assert e.value.status == qc.QC_ERR_INVALID_ARG
    b.table.state[1] = 0
    run(b)


def test_more_queries_than_the_call_says():
    b = Batch(19, [5, 60], [1, 3], [], 2, 2, 64, 16)
    out = torch.full_like(b.q, 3.0)
    b.call(max_queries=2, out=out)
    assert (out == 3).all() and int(b.table.state[1]) == qc.QC_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1])
def test_keys_of_pages_that_are_none_count_as_absent(bad):
    b = Batch(20, [70, 130], [1, 1], [(0, 2, 100)], 2, 2, 128, 16)
    gone = [(b.table, int(b.ids[1]), 3, b.keys, b.values, 1), (b.shared[0], int(b.shared_ids[0]), 6, b.shared[2], b.shared[3], 0)]
    for t, row, col, keys, values, i in gone:
        t.pages[row, col] = bad
        keep = torch.tensor([j // 16 != col for j in range(len(keys[i]))], device=DEV)
        keys[i], values[i] = keys[i][keep], values[i][keep]
    b.lens[1], b.groups[0] = len(b.keys[1]), (0, 2, len(b.shared[2][0]))
    out, lse = b.call()
    assert int(b.table.state[1]) == qc.QC_ERR_BAD_PAGE
    b.check(out, lse)


def test_lengths_beyond_the_table_are_cut():
    b = Batch(21, [40, 64], [1, 1], [(0, 1, 20)], 1, 2, 64, 16)
    room = b.table.pages.shape[1] * 16
    b.table.lens[b.ids[0].long()] = -5
    b.table.lens[b.ids[1].long()] = room + 1000
    out, lse = b.call()
    # (the pages behind the 64 tokens are none, so their keys are absent)
    assert int(b.table.state[1]) in (qc.QC_ERR_PLAN, qc.QC_ERR_BAD_PAGE)
    b.keys[0], b.values[0], b.lens[0] = b.keys[0][:0], b.values[0][:0], 0
    b.check(out, lse)


# ---- captured, on other streams, one after the other -----------------------------------------------------------------

def test_replays_follow_the_lengths():
    """A captured step whose sequences grow from replay to replay, with another captured batch between."""
    b, other = Batch(22, [3, 60, 200], [1, 1, 1], [(0, 2, 90)], 2, 4, 128, 16), Batch(23, [500, 2], [2, 1], [(0, 2, 1000)], 2, 4, 128, 16)
    want_other = run(other)
    run(b)
    graphs = []
    for x in (b, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = x.call()
        graphs.append((graph, got))
    full = list(b.lens)
    for cut in ([3, 60, 200], [1, 17, 64], [0, 1, 130], [3, 59, 199]):
        for i, n in enumerate(cut):
            b.table.lens[b.ids[i].long()] = n
        graphs[0][0].replay()
        graphs[1][0].replay()
        keys, values = b.keys, b.values
        b.keys, b.values, b.lens = [k[:n] for k, n in zip(keys, cut)], [v[:n] for v, n in zip(values, cut)], cut
        b.check(*graphs[0][1])
        b.keys, b.values, b.lens = keys, values, full
        assert torch.equal(graphs[1][1][0], want_other[0]) and torch.equal(graphs[1][1][1], want_other[1])


def test_captured_steps_that_share_their_memory():
    """Two graphs of one memory pool, whose workspaces may be the same bytes, replayed in turn."""
    batches = Batch(31, [300] * 6, [1] * 6, [(0, 6, 900)], 4, 4, 128, 16), Batch(32, [20, 700], [2, 3], [(0, 2, 64)], 4, 4, 128, 16)
    want = [run(b) for b in batches]
    graphs, got = [torch.cuda.CUDAGraph() for _ in batches], []
    for graph, b in zip(graphs, batches):
        with torch.cuda.graph(graph, pool=graphs[0].pool() if got else None):
            got.append(b.call())
    for turn in (0, 1, 1, 0, 1):
        for x in got[turn]:
            x.zero_()
        graphs[turn].replay()
        assert torch.equal(got[turn][0], want[turn][0]) and torch.equal(got[turn][1], want[turn][1])


def test_two_calls_on_two_streams_at_once():
    a, b = Batch(24, [900] * 8, [1] * 8, [(0, 8, 3000)], 4, 4, 128, 16), Batch(25, [40] * 30, [1] * 30, [(3, 30, 700)], 4, 4, 128, 16)
    want = run(a), run(b)
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(sides[i]):
                got[i].append(x.call())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]) for out, lse in got[i])


# ---- what does not fit on the host -----------------------------------------------------------------------------------

@pytest.mark.parametrize("change", [
    dict(seq_ids=lambda b: b.ids.long()), dict(seq_ids=lambda b: b.ids[:2]), dict(starts=lambda b: b.starts[:3]), dict(starts=lambda b: b.starts.cpu()), dict(max_queries=lambda b: 0),
    dict(max_queries=lambda b: qc.QC_PAGED_MAX_QUERIES + 1), dict(scale=lambda b: -1.0), dict(scale=lambda b: math.inf), dict(groups=lambda b: b.group_starts.long()), dict(groups=lambda b: None),
    dict(shared_ids=lambda b: b.shared_ids[:1]), dict(shared=lambda b: None), dict(out=lambda b: b.q), dict(out=lambda b: b.q_shared), dict(out=lambda b: torch.zeros(4, 4, 64, device=DEV)),
    dict(out=lambda b: torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV)), dict(status=lambda b: torch.zeros(2, dtype=torch.int32, device=DEV)),
    dict(own=lambda b: b.stream()._replace(q=b.q.float())), dict(own=lambda b: b.stream()._replace(q=b.q[:, :3])), dict(own=lambda b: b.stream()._replace(k_pool=b.pools[0][:1])),
    dict(own=lambda b: b.stream()._replace(k_pool=b.pools[0].float())), dict(own=lambda b: b.stream()._replace(pages=b.table.pages[0])), dict(own=lambda b: b.stream()._replace(lens=b.table.lens[:2])),
    dict(shared=lambda b: b.shared_stream()._replace(q=b.q[:2])), dict(shared=lambda b: b.shared_stream()._replace(k_pool=b.shared[1][0][:, :1].contiguous(), v_pool=b.shared[1][1][:, :1].contiguous())),
])
def test_what_does_not_fit_is_refused(change):
    b = Batch(26, [5, 60, 7], [1, 2, 1], [(0, 2, 9), (2, 3, 70)], 2, 2, 64, 16, lazy=True)
    run(b)
    with pytest.raises((ValueError, qc.QcError)):
        b.call(**{k: make(b) for k, make in change.items()})


def test_nothing_to_do():
    b = Batch(27, [5, 60], [1, 1], [(0, 2, 9)], 2, 2, 64, 16)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    q = b.q[:0]
    out, lse = b.call(own=b.stream()._replace(q=q), shared=b.shared_stream()._replace(q=q), seq_ids=none, starts=none.new_zeros(1), groups=none.new_zeros(1), shared_ids=none)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    # sequences without queries, and a list of groups without any
    out, lse = b.call(own=b.stream()._replace(q=b.q[:1]), shared=b.shared_stream()._replace(q=b.q[:1]), starts=torch.tensor([0, 0, 1], dtype=torch.int32, device=DEV), groups=none.new_zeros(1), shared_ids=none)
    check_rows_of(out, lse, [(b.q[:1], b.keys[1], b.values[1], torch.tensor([60], device=DEV))], 2, b.scale, "sequence 1")


# ---- as they are used ------------------------------------------------------------------------------------------------

def test_questions_about_two_images_from_projection_to_attention():
    """Images are appended once, then every step normalises and turns queries and keys, appends, and attends over image and text."""
    g = gen(30)
    hkv, group, d, page, n = 2, 3, 128, 16, 5
    hq = hkv * group
    images, texts = paged.PageTable.empty(3, 20, page, 40), paged.PageTable.empty(8, 6, page, 30)
    pools = {name: [paged.empty_pool(hkv, d, page, t.free.numel()) for _ in "kv"] for name, t in (("image", images), ("text", texts))}
    rot, freqs, axes = rotation(d, 3, g)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).bfloat16().to(DEV) for _ in "qk")
    turn = dict(rotation=rot, q_norm=wq, k_norm=wk, eps=1e-6)
    sizes, image_rows = [150, 97], torch.tensor([2, 0], dtype=torch.int32, device=DEV)
    _, slots = paged.table_extend(images, torch.tensor(sizes, dtype=torch.int32, device=DEV), seq_ids=image_rows, max_slots=sum(sizes))
    x = rows(sum(sizes), 2 * hkv, d, g).to(DEV)
    patches = torch.randint(0, 40, (3, sum(sizes)), generator=g, dtype=torch.int32).to(DEV)
    paged.append(*pools["image"], slots, x[:, :hkv], x[:, hkv:], positions=patches, **turn)
    image_keys = paged.rotate(None, x[:, :hkv], patches, rot, k_norm=wk)[1].split(sizes)
    image_values = x[:, hkv:].split(sizes)
    ids, groups = torch.tensor([6, 1, 3, 0, 4], dtype=torch.int32, device=DEV), torch.tensor([1, 3, 5], dtype=torch.int32, device=DEV)      # the first asks about none
    keys, values = [[] for _ in range(n)], [[] for _ in range(n)]
    for step in range(4):
        new = torch.tensor([[9, 20, 1, 33, 17], [1] * 5, [3, 1, 2, 1, 1], [1] * 5][step], dtype=torch.int32, device=DEV)
        total = int(new.sum())
        starts, slots = paged.table_extend(texts, new, seq_ids=ids, max_slots=total + 2)
        fused = rows(total + 2, hq + 2 * hkv, d, g).to(DEV)                          # two tokens of padding
        positions = torch.randint(0, 5000, (3, total + 2), generator=g, dtype=torch.int32).to(DEV)
        q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        turned_k = paged.rotate(None, k, positions, rot, k_norm=wk)[1]
        q = paged.append(*pools["text"], slots, k, v, q=q, positions=positions, **turn)
        out, lse = paged.attend(paged.Stream(q, *pools["text"], texts.pages, texts.lens), shared=paged.Stream(q, *pools["image"], images.pages, images.lens), groups=groups,
                                shared_ids=image_rows, seq_ids=ids, starts=starts, max_queries=int(new.max()), status=texts.state[1:2])
        texts.check()
        begin = starts.tolist()
        for i in range(n):
            a, b = begin[i], begin[i + 1]
            keys[i].append(turned_k[a:b])
            values[i].append(v[a:b])
            k_all, v_all = torch.cat(keys[i]), torch.cat(values[i])
            parts = [(q[a:b], k_all, v_all, len(k_all) - (b - a - 1) + torch.arange(b - a, device=DEV))]
            if i:
                j = 0 if i < 3 else 1
                parts.insert(0, (q[a:b], image_keys[j], image_values[j], torch.full((b - a,), sizes[j], device=DEV)))
            check_rows_of(out[a:b], lse[a:b], parts, group, 1 / math.sqrt(d), (step, i))
