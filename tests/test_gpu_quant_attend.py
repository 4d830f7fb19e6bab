"""Attention over a cache in 4 bits against the oracle in 64 bits on what the cache holds, element by element within the
bound that ``quant_util.bound`` derives, and the three calls together as a step makes them."""

import math
import random

import numpy as np
import pytest
import torch

from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

from quant_util import DEV, check_attend, check_attend_torch, fill, gen, held, held_torch, rows

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """One stream: a table whose rows are listed in an order of their own, pools whose unused bytes are NaN rows."""

    def __init__(self, lens, heads, head_dim, page, seed, ids=None, slack=3):
        g = gen(seed)
        self.lens, self.page, self.heads, self.head_dim = lens, page, heads, head_dim
        n = len(lens) + 2
        self.ids = i32(ids if ids is not None else torch.randperm(n, generator=g)[: len(lens)].tolist())
        n_pages = sum(-(-x // page) for x in lens) + slack
        self.table = quant.PageTable.empty(n, max(-(-x // page) for x in lens) + 2, page, n_pages)
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table.free.copy_(order.to(DEV))
        self.pools = [quant.empty_pool(heads, head_dim, page, n_pages) for _ in "kv"]
        for p in self.pools:
            p.fill_(0xFF)                         # lo and r are no numbers
        self.k, self.v = [rows(x, heads, head_dim, g) for x in lens], [rows(x, heads, head_dim, g) for x in lens]
        fill(self.table, self.ids, lens, page, self.pools, self.k, self.v)
        self.k_held, self.v_held = [held(x) for x in self.k], [held(x) for x in self.v]

    def stream(self, q):
        return quant.Stream(q, self.pools[0], self.pools[1], self.table.pages, self.table.lens)


def queries(counts, heads, head_dim, seed, size=1.0):
    g = gen(seed + 77)
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    return starts, (torch.randn(starts[-1], heads, head_dim, generator=g) * size).bfloat16()


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads,group,lens", [
    (1, 1, [1]), (2, 1, [63, 64, 65]), (1, 8, [15, 16, 17, 0]), (2, 7, [257, 1, 130]), (3, 5, [700, 33]), (1, 3, [2100]), (1, 16, [90, 300]),
], ids=lambda x: str(x).replace(" ", ""))
def test_one_query_each(page, head_dim, heads, group, lens):
    c = Cache(lens, heads, head_dim, page, 11 * page + head_dim + heads)
    starts, q = queries([1] * len(lens), heads * group, head_dim, page)
    status = i32([0])
    out, lse = quant.attend(c.stream(q.to(DEV)), heads, page, seq_ids=c.ids, status=status)
    check_attend(out, lse, starts, None, lens, q, c.k_held, c.v_held, group, head_dim ** -0.5)
    assert int(status) == qc.QC_OK


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("head_dim,page", [(64, 32), (128, 16)])
@pytest.mark.parametrize("heads,group,lens,counts", [
    (1, 1, [5, 70, 3], [5, 2, 5]), (2, 4, [129, 64, 0, 17], [2, 0, 1, 3]), (1, 7, [200, 66], [16, 1]), (1, 16, [40, 129], [3, 2]),
    (2, 1, [2, 1, 300], [4, 3, 16]),
], ids=lambda x: str(x).replace(" ", ""))
def test_several_queries_see_no_token_behind_their_own(causal, head_dim, page, heads, group, lens, counts):
    c = Cache(lens, heads, head_dim, page, 5 * page + head_dim + heads)
    starts, q = queries(counts, heads * group, head_dim, page + group)
    out = torch.full((starts[-1] + 2, heads * group, head_dim), 9.0, dtype=torch.bfloat16, device=DEV)
    padded = torch.cat([q, torch.full((2, heads * group, head_dim), float("nan")).bfloat16()])
    got, lse = quant.attend(c.stream(padded.to(DEV)), heads, page, seq_ids=c.ids, starts=i32(starts), max_queries=max(counts), causal=causal, out=out)
    assert got is out and (out[starts[-1]:] == 9.0).all()          # rows behind the last sequence
    check_attend(out, lse, starts, None, lens, q, c.k_held, c.v_held, group, head_dim ** -0.5, causal=causal)


@pytest.mark.parametrize("head_dim,page", [(64, 16), (128, 64), (128, 16)])
@pytest.mark.parametrize("heads,group,text,vis,counts", [
    (2, 1, [35, 0, 7], [576, 130, 0], [1, 1, 1]), (1, 7, [3, 99], [64, 1], [1, 1]), (1, 4, [10, 2, 0], [100, 65, 5], [3, 2, 1]),
], ids=lambda x: str(x).replace(" ", ""))
def test_two_streams_with_a_query_each_have_one_softmax(head_dim, page, heads, group, text, vis, counts):
    t = Cache(text, heads, head_dim, page, 3 * page + head_dim)
    v = Cache(vis, heads, head_dim, page, 4 * page + head_dim, ids=t.ids.tolist())
    starts, q = queries(counts, heads * group, head_dim, page)
    _, qv = queries(counts, heads * group, head_dim, page + 1, size=0.01 if group == 4 else 1.5)
    out, lse = quant.attend(t.stream(q.to(DEV)), heads, page, visual=v.stream(qv.to(DEV)), seq_ids=t.ids, starts=i32(starts), max_queries=max(counts))
    check_attend(out, lse, starts, None, text, q, t.k_held, t.v_held, group, head_dim ** -0.5, visual=(qv, v.k_held, v.v_held))


def test_a_leader_s_keys_under_values_of_another_pool():
    """GLA: both streams' queries and keys are the leader's, the values the layer's own."""
    lead, own = Cache([150, 40], 2, 128, 16, 1, ids=[0, 1]), Cache([150, 40], 2, 128, 16, 2, ids=[0, 1])
    starts, q = queries([1, 1], 4, 128, 0)
    own.table.pages.copy_(lead.table.pages)      # one table serves all layers
    order = torch.cat([lead.table.pages[i][: -(-n // 16)] for i, n in enumerate([150, 40])]).long()
    pool = torch.full_like(own.pools[1], 0xFF)
    slots = []
    for i, n in enumerate([150, 40]):
        pos = torch.arange(n, device=DEV)
        slots.append(lead.table.pages[i].long()[pos // 16] * 16 + pos % 16)
    assert len(order) == 13
    quant.append(None, pool, torch.cat(slots).to(torch.int32), None, torch.cat(own.v).to(DEV), 16)
    out, lse = quant.attend(quant.Stream(q.to(DEV), lead.pools[0], pool, lead.table.pages, lead.table.lens), 2, 16, seq_ids=lead.ids)
    check_attend(out, lse, starts, None, [150, 40], q, lead.k_held, own.v_held, 2, 128 ** -0.5)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("size,scale", [(30.0, 0.0), (1e-3, 0.0), (1e4, 1e-3), (1.0, 2.0), (2.0 ** 60, 2.0 ** -62)])
def test_queries_and_scales_of_other_magnitudes(head_dim, size, scale):
    c = Cache([300, 77], 1, head_dim, 32, 8)
    starts, q = queries([1, 1], 4, head_dim, 5, size=size)
    out, lse = quant.attend(c.stream(q.to(DEV)), 1, 32, seq_ids=c.ids, scale=scale)
    check_attend(out, lse, starts, None, [300, 77], q, c.k_held, c.v_held, 4, scale or head_dim ** -0.5)


def test_values_whose_ranges_are_far_apart_and_rows_without_range():
    c = Cache([200], 1, 128, 16, 4, ids=[1])
    g = gen(1)
    v = c.v[0].clone()
    v[::3] = (v[::3].float() * 2.0 ** torch.randint(-12, 12, (67, 1, 1), generator=g)).bfloat16()
    v[5], v[6], v[7] = 3.0, 0.0, -1000.0
    k = c.k[0].clone()
    k[9], k[10] = 0.5, 0.0
    slots = c.table.pages[1].long()[torch.arange(200, device=DEV) // 16] * 16 + torch.arange(200, device=DEV) % 16
    quant.append(c.pools[0], c.pools[1], slots.to(torch.int32), k.to(DEV), v.to(DEV), 16)
    starts, q = queries([1], 8, 128, 2)
    out, lse = quant.attend(c.stream(q.to(DEV)), 1, 16, seq_ids=c.ids)
    check_attend(out, lse, starts, None, [200], q, [held(k)], [held(v)], 8, 128 ** -0.5)


def test_what_is_no_number_counts_where_it_is_seen():
    """A NaN row of K or V makes the outputs NaN of the queries that see it, and of no others."""
    for which in (0, 1):
        c = Cache([90, 70], 1, 64, 16, 6, ids=[0, 1])
        bad = (c.k if which == 0 else c.v)[0][88:89].clone()
        bad[0, 0, 3] = float("inf")
        slot = int(c.table.pages[0, 88 // 16]) * 16 + 88 % 16
        pools = [None, None]
        pools[which] = c.pools[which]
        given = [bad.to(DEV) if i == which else None for i in range(2)]
        quant.append(pools[0], pools[1], i32([slot]), given[0], given[1], 16)
        starts, q = queries([3, 2], 4, 64, 3)
        out, lse = quant.attend(c.stream(q.to(DEV)), 1, 16, seq_ids=c.ids, starts=i32(starts), max_queries=3)
        # query 0 sees 88 tokens (not the bad one at 88), queries 1 and 2 see it
        assert torch.isnan(out[1:3].float()).all() and torch.isfinite(out[[0, 3, 4]].float()).all()
        assert torch.isnan(lse[1:3]).all() if which == 0 else torch.isfinite(lse).all()
        k_held, v_held = [{n: a[:88] for n, a in c.k_held[0].items()}], [{n: a[:88] for n, a in c.v_held[0].items()}]
        check_attend(out[:1], lse[:1], [0, 1], None, [88], q[:1], k_held, v_held, 4, 64 ** -0.5)
        check_attend(out[3:], lse[3:], [0, 2], None, [70], q[3:], c.k_held[1:], c.v_held[1:], 4, 64 ** -0.5)


def test_scores_that_are_infinite_and_queries_that_are_no_numbers():
    c = Cache([130], 1, 64, 16, 6, ids=[0])
    q = torch.ones(1, 3, 64)
    q[0, 1, 5] = float("nan")
    out, lse = quant.attend(c.stream(q.bfloat16().to(DEV)), 1, 16, seq_ids=c.ids)
    assert torch.isfinite(out[0, [0, 2]].float()).all() and torch.isnan(out[0, 1].float()).all() and torch.isnan(lse[0, 1])
    check_attend(out[:, [0]], lse[:, [0]], [0, 1], None, [130], q[:, [0]].bfloat16(), c.k_held, c.v_held, 1, 64 ** -0.5)


def test_device_numbers_out_of_range_are_reported_and_not_followed():
    c = Cache([40, 100, 60], 1, 64, 16, 6, ids=[0, 1, 2])
    starts, q = queries([1, 2, 1], 2, 64, 3)
    qd = q.to(DEV)

    def run(ids=(0, 1, 2), begin=starts, most=2):
        status, out = i32([0]), torch.full((4, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
        got, lse = quant.attend(c.stream(qd), 1, 16, seq_ids=i32(list(ids)), starts=i32(list(begin)), max_queries=most, out=out, status=status)
        return int(status), got, lse

    def fine(out, lse, which, held_len=None):
        a = [(0, 1), (1, 3), (3, 4)][which]
        n = [40, 100, 60][which]
        check_attend(out[a[0]:a[1]], lse[a[0]:a[1]], [0, a[1] - a[0]], None, [n], q[a[0]:a[1]], [c.k_held[which]], [c.v_held[which]], 2, 64 ** -0.5)

    status, out, lse = run()
    assert status == 0
    for i in range(3):
        fine(out, lse, i)
    for ids in ((0, 5, 2), (0, -1, 2)):
        status, out, lse = run(ids=ids)
        assert status == qc.QC_ERR_INVALID_ARG and (out[1:3] == 9.0).all()
        fine(out, lse, 0), fine(out, lse, 2)
    for begin in ((0, 1, 3, 900), (0, 1, 3, 2), (0, 1, 3, -4)):
        status, out, lse = run(begin=begin)
        assert status == qc.QC_ERR_INVALID_ARG and (out[3] == 9.0).all()
        fine(out, lse, 0), fine(out, lse, 1)
    status, out, lse = run(most=1)
    assert status == qc.QC_ERR_INVALID_ARG and (out[1:3] == 9.0).all()
    # a page that is none: its keys are absent
    saved = c.table.pages.clone()
    for bad in (-1, 1 << 30, c.pools[0].shape[0]):
        c.table.pages[1, 2] = bad
        status, out, lse = run()
        assert status == qc.QC_ERR_BAD_PAGE
        fine(out, lse, 0), fine(out, lse, 2)
        keep = np.r_[0:32, 48:100]
        cut = lambda h: [{n: a[keep] for n, a in h.items()}]
        check_attend(out[1:3], lse[1:3], [0, 2], None, [84], q[1:3], cut(c.k_held[1]), cut(c.v_held[1]), 2, 64 ** -0.5)
    c.table.pages.copy_(saved)
    for bad in (-7, 1 << 30):
        c.table.lens[2] = bad
        status, out, lse = run()
        assert status in (qc.QC_ERR_PLAN, qc.QC_ERR_BAD_PAGE)
        fine(out, lse, 0), fine(out, lse, 1)
        if bad < 0:
            assert (out[3] == 0).all() and (lse[3] == -math.inf).all()


def test_strided_queries_and_one_query_for_all():
    c = Cache([100, 30, 64], 2, 128, 16, 6)
    starts, q = queries([1, 1, 1], 8, 128, 3)
    fused = torch.zeros(3, 12, 128, dtype=torch.bfloat16, device=DEV)
    fused[:, 2:10] = q.to(DEV)
    out, lse = quant.attend(c.stream(fused[:, 2:10]), 2, 16, seq_ids=c.ids)
    check_attend(out, lse, starts, None, c.lens, q, c.k_held, c.v_held, 4, 128 ** -0.5)
    one = q[:1].to(DEV).expand(3, 8, 128)
    out, lse = quant.attend(c.stream(one), 2, 16, seq_ids=c.ids)
    check_attend(out, lse, starts, None, c.lens, q[:1].expand(3, 8, 128), c.k_held, c.v_held, 4, 128 ** -0.5)


@pytest.mark.parametrize("head_dim,heads,group,n,page", [(128, 2, 4, 20001, 64), (64, 1, 1, 33333, 16), (128, 1, 16, 12345, 32)])
def test_long_sequences_against_torch_in_64_bits(head_dim, heads, group, n, page):
    """Values with a mean, so that what long sums lose would show; the same bound, from device arithmetic in 64 bits."""
    g = gen(n)
    table = quant.PageTable.empty(1, -(-n // page), page, -(-n // page))
    pools = [quant.empty_pool(heads, head_dim, page, -(-n // page)) for _ in "kv"]
    k, v = (torch.randn(n, heads, head_dim, generator=g) + m for m in (0.0, 0.3))
    _, slots = quant.table_extend(table, i32([n]), max_slots=n)
    quant.append(pools[0], pools[1], slots, k.bfloat16().to(DEV), v.bfloat16().to(DEV), page)

    def split(x):
        x = x.bfloat16().double().to(DEV)
        lo, hi = x.min(-1).values, x.max(-1).values
        r = (15 / (hi - lo)).float().bfloat16().double()     # (a span of two bf16 numbers; ties of the second rounding apart)
        codes = torch.round((x - lo[..., None]) * r[..., None])
        return lo, 1 / r, codes

    (kl, ks, kc), (vl, vs, vc) = split(k), split(v)
    back = quant.read(pools[0], pools[1], slots, heads, head_dim, page)
    for b, (lo, s, c) in zip(back, ((kl, ks, kc), (vl, vs, vc))):
        assert ((b.double() - (lo[..., None] + s[..., None] * c)).abs() <= 2.0 ** -8 * ((lo[..., None] + s[..., None] * c).abs() + 2.0 ** -14 * (lo.abs() + 15 * s)[..., None])).all()
    q = torch.randn(1, heads * group, head_dim, generator=g).bfloat16()
    out, lse = quant.attend(quant.Stream(q.to(DEV), pools[0], pools[1], table.pages, table.lens), heads, page)
    for h in range(heads * group):
        j, x = h // group, q[0, h].double().to(DEV)
        logit = (kl[:, j, None] + ks[:, j, None] * kc[:, j]) @ x * head_dim ** -0.5
        want_lse = torch.logsumexp(logit, 0)
        w = torch.exp(logit - want_lse)
        want = w @ (vl[:, j, None] + vs[:, j, None] * vc[:, j])
        small = (x.abs() < 2.0 ** -9 * x.abs().max()).double()
        part = ((kc[:, j] @ x.abs()) * ks[:, j] + kl[:, j].abs() * x.abs().sum()) * (head_dim + 12) * 2.0 ** -23
        e = ((part + (kc[:, j] @ small) * ks[:, j] * 2.0 ** -17 * x.abs().max()).max() * head_dim ** -0.5).item()
        mass = w @ ((vl[:, j] + 8 * vs[:, j]).abs()[:, None] + vs[:, j, None] * (vc[:, j] - 8).abs())
        rel = 2 * e + 2.0 ** -21 + (n + 64) * 2.0 ** -23
        assert ((out[0, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * rel) * mass).all()
        # the bound above allows for the worst; roundings of either sign leave far less: their root mean square
        err = ((out[0, h].double() - want).norm() / want.norm()).item()
        assert err <= 2.0 ** -8, err
        assert abs(lse[0, h].item() - want_lse.item()) <= e + 2.0 ** -20 + (n + 64) * 2.0 ** -23


@pytest.mark.parametrize("seqs,heads,group,head_dim,page,low,high,most", [
    (70, 2, 1, 128, 16, 1, 130, 1),          # more sequences than one warp counts, units that are not cut
    (300, 1, 8, 64, 32, 0, 700, 2),
    (2048, 1, 1, 128, 16, 0, 90, 1),         # the most sequences
    (2048, 1, 3, 64, 64, 0, 90, 2),
    (100, 4, 4, 128, 16, 1, 3000, 1),        # ranges of one warp, cut
    (60, 2, 1, 64, 16, 900, 5000, 3),
    (24, 3, 2, 128, 32, 1, 6000, 1),
    (9, 2, 16, 128, 16, 2000, 9000, 1),      # sixteen rows to a unit
    (5, 1, 8, 64, 16, 100, 9000, 16),        # the most queries, in units of sixteen rows
    (7, 1, 5, 128, 64, 100, 9000, 15),       # and in units of eight
    (2, 2, 1, 128, 64, 40000, 41000, 1),     # few long ones: a unit in the ranges of many teams
    (1, 1, 16, 64, 16, 60000, 60000, 1),
    (1, 1, 1, 128, 16, 30001, 30001, 1),
    (1, 1, 4, 128, 32, 50007, 50007, 2),
    (130, 8, 1, 128, 16, 512, 512, 1),
])
def test_batches_of_many_kinds_against_torch_in_64_bits(seqs, heads, group, head_dim, page, low, high, most):
    rng, g = random.Random(seqs + high), gen(seqs + high)
    lens = [rng.randint(low, high) for _ in range(seqs)]
    counts = [rng.randint(0 if seqs > 9 else 1, most) if most > 1 else 1 for _ in range(seqs)]
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    total = sum(lens)
    table = quant.PageTable.empty(seqs, max(1, -(-high // page)), page, sum(-(-n // page) for n in lens) + 1)
    pools = [quant.empty_pool(heads, head_dim, page, table.free.numel()) for _ in "kv"]
    for p in pools:
        p.fill_(0xFF)
    ids = i32(torch.randperm(seqs, generator=g).tolist())
    k, v = (rows(total, heads, head_dim, g).to(DEV) for _ in "kv")
    _, slots = quant.table_extend(table, i32(lens), seq_ids=ids, max_slots=total)
    quant.append(pools[0], pools[1], slots, k, v, page)
    q = torch.randn(max(1, starts[-1]), heads * group, head_dim, generator=g).bfloat16().to(DEV)
    status = i32([0])
    stream = quant.Stream(q, pools[0], pools[1], table.pages, table.lens)
    out, lse = quant.attend(stream, heads, page, seq_ids=ids, starts=i32(starts), max_queries=most, status=status)
    again, lse_again = quant.attend(stream, heads, page, seq_ids=ids, starts=i32(starts), max_queries=most)
    assert int(status) == qc.QC_OK
    used = starts[-1]
    assert torch.equal(out[:used], again[:used]) and torch.equal(lse[:used], lse_again[:used])
    first = [0]
    for n in lens:
        first.append(first[-1] + n)
    k_held, v_held = held_torch(k), held_torch(v)
    seq_of = torch.repeat_interleave(torch.arange(seqs), torch.tensor(counts))
    picked = list(range(used)) if used * max(lens) * head_dim < 2e7 else sorted(rng.sample(range(used), max(1, min(used, int(2e7 / (max(lens) * head_dim))))))
    for h in range(heads * group):
        if heads * group > 8 and h not in (0, 1, heads * group - 1) and rng.random() < 0.5:
            continue
        j = h // group
        for at in range(0, len(picked), max(1, int(2e7 / (max(lens + [1]) * head_dim)))):
            part = picked[at: at + max(1, int(2e7 / (max(lens + [1]) * head_dim)))]
            s = [int(seq_of[t]) for t in part]
            seen = [max(0, lens[i] - (starts[i + 1] - 1 - t)) for t, i in zip(part, s)]
            width = max(seen + [1])
            place = torch.tensor([first[i] for i in s])[:, None] + torch.arange(width)
            place = place.clamp_(max=max(0, total - 1)).to(DEV)
            cut = lambda a: {name: x[place, j] for name, x in a.items()}
            check_attend_torch(out[part, h], lse[part, h], q[part, h], cut(k_held), cut(v_held), torch.tensor(seen, device=DEV), head_dim ** -0.5)


@pytest.mark.parametrize("seqs,heads,group,head_dim,tokens", [(1, 1, 1, 128, 30000), (3, 2, 4, 64, 9001), (30, 8, 1, 128, 1900), (40, 4, 16, 64, 700)])
def test_a_captured_call_gives_the_same_bits_each_time(seqs, heads, group, head_dim, tokens):
    g, page = gen(tokens), 32
    per = -(-tokens // page)
    table = quant.PageTable.empty(seqs, per, page, seqs * per)
    pools = [torch.empty_like(quant.empty_pool(heads, head_dim, page, seqs * per)) for _ in "kv"]
    _, slots = quant.table_extend(table, torch.full((seqs,), tokens, dtype=torch.int32, device=DEV), max_slots=seqs * tokens)
    rows_ = torch.randn(seqs * tokens, heads, head_dim, generator=g).bfloat16().to(DEV)
    quant.append(pools[0], pools[1], slots, rows_, rows_.flip(0).contiguous(), page)
    q = torch.randn(seqs, heads * group, head_dim, generator=g).bfloat16().to(DEV)
    stream = quant.Stream(q, pools[0], pools[1], table.pages, table.lens)
    want, want_lse = quant.attend(stream, heads, page)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [quant.attend(stream, heads, page) for _ in range(4)]
    for _ in range(50):
        for out, lse in outs:
            out.fill_(7)
        graph.replay()
        for out, lse in outs:
            assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("seqs,heads", [(1, 2), (40, 1), (100, 1)])      # one sequence too long, a batch too large, one of more sequences than a warp counts
def test_a_batch_that_is_too_much_for_one_call_is_left_alone(seqs, heads):
    pages, lens = torch.full((1, 1 << 22), -1, dtype=torch.int32, device=DEV), i32([1 << 28])
    pool = quant.empty_pool(heads, 64, 64, 1).zero_()
    q, status = torch.ones(seqs, heads, 64, dtype=torch.bfloat16, device=DEV), i32([0])
    out = torch.full_like(q, 3)
    quant.attend(quant.Stream(q, pool, pool, pages, lens), heads, 64, seq_ids=i32([0] * seqs), out=out, status=status)
    assert int(status) == qc.QC_ERR_PLAN and bool((out == 3).all())


def test_pages_behind_four_gigabytes():
    heads, head_dim, page = 32, 128, 64
    per = heads * page * (head_dim // 2 + 4)
    n_pages = (5 << 30) // per
    pools = [quant.empty_pool(heads, head_dim, page, n_pages) for _ in "kv"]
    g = gen(4)
    k, v = rows(100, heads, head_dim, g), rows(100, heads, head_dim, g)
    pages, lens = i32([[n_pages - 1, n_pages - 2]]), i32([100])
    slots = torch.cat([torch.arange(64) + (n_pages - 1) * 64, torch.arange(36) + (n_pages - 2) * 64]).to(torch.int32).to(DEV)
    quant.append(pools[0], pools[1], slots, k.to(DEV), v.to(DEV), page)
    q = torch.randn(1, heads, head_dim, generator=g).bfloat16()
    out, lse = quant.attend(quant.Stream(q.to(DEV), pools[0], pools[1], pages, lens), heads, page)
    check_attend(out, lse, [0, 1], None, [100], q, [held(k)], [held(v)], 1, head_dim ** -0.5)


# ---- the calls together -------------------------------------------------------------------------------

class Step:
    """What a program that decodes keeps: a text and a visual stream, two layers of which the second is lazy (VLA_QC:
    it scores the visual keys of the first with the first's query and has no visual K of its own)."""

    def __init__(self, seqs, heads, group, head_dim, page, room):
        self.seqs, self.heads, self.group, self.head_dim, self.page = seqs, heads, group, head_dim, page
        per = -(-room // page)
        self.text, self.visual = (quant.PageTable.empty(seqs, per, page, seqs * per) for _ in range(2))
        make = lambda: quant.empty_pool(heads, head_dim, page, seqs * per)
        self.kt, self.vt, self.vv, self.kv = [make(), make()], [make(), make()], [make(), make()], make()

    def prompt(self, lens, vis, rows_t, rows_v):
        _, st = quant.table_extend(self.text, i32(lens), max_slots=sum(lens))
        _, sv = quant.table_extend(self.visual, i32(vis), max_slots=sum(vis))
        for l in range(2):
            quant.append(self.kt[l], self.vt[l], st, rows_t[l][0].to(DEV), rows_t[l][1].to(DEV), self.page)
        quant.append(self.kv, self.vv[0], sv, rows_v[0][0].to(DEV), rows_v[0][1].to(DEV), self.page)
        quant.append(None, self.vv[1], sv, None, rows_v[1][1].to(DEV), self.page)

    def decode(self, q, k, v, n_new, tokens, most):
        """q, k, v: [layer][tokens, heads, head_dim] on the device."""
        starts, slots = quant.table_extend(self.text, n_new, max_slots=tokens)
        outs = []
        for l in range(2):
            quant.append(self.kt[l], self.vt[l], slots, k[l], v[l], self.page)
            outs.append(quant.attend(quant.Stream(q[l], self.kt[l], self.vt[l], self.text.pages, self.text.lens), self.heads, self.page,
                                     visual=quant.Stream(q[0], self.kv, self.vv[l], self.visual.pages, self.visual.lens),
                                     starts=starts, max_queries=most, status=self.text.state[1:2]))
        return outs


@pytest.mark.parametrize("head_dim,group,captured", [(64, 1, False), (128, 4, False), (128, 1, True), (64, 7, True)])
def test_a_run_of_steps_with_drafts_turned_down(head_dim, group, captured):
    seqs, heads, page, most = 3, 2, 16, 4
    g = gen(head_dim + group)
    s = Step(seqs, heads, group, head_dim, page, 160)
    text, vis = [20, 3, 45], [64, 0, 33]
    R = lambda n: rows(n, heads, head_dim, g)
    pt, pv = [(R(sum(text)), R(sum(text))) for _ in range(2)], [(R(sum(vis)), R(sum(vis))) for _ in range(2)]
    s.prompt(text, vis, pt, pv)
    cut = lambda x, ns: list(torch.split(x, ns))
    kept = [[cut(pt[l][i], text) for i in range(2)] for l in range(2)]        # [layer][k or v][sequence]
    vis_held = [[[held(x) for x in cut(pv[l][i], vis)] for i in range(2)] for l in range(2)]
    tokens = seqs * most
    dev = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)
    q, k, v = ([dev(tokens, n, head_dim) for _ in range(2)] for n in (heads * group, heads, heads))
    n_new, keep = dev(seqs, dtype=torch.int32), dev(seqs, dtype=torch.int32)
    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        saved = [t.clone() for t in (s.text.pages, s.text.lens, s.text.free, s.text.state)]
        with torch.cuda.stream(side):
            s.decode(q, k, v, n_new, tokens, most)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip((s.text.pages, s.text.lens, s.text.free, s.text.state), saved):
            a.copy_(b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = s.decode(q, k, v, n_new, tokens, most)
            quant.table_trim(s.text, keep)
    lens = list(text)
    rng = random.Random(4)
    for step in range(6):
        counts = [rng.randint(0 if step else 1, most) for _ in range(seqs)]
        accepted = [rng.randint(min(c, 1), c) for c in counts]
        total = sum(counts)
        new = [[torch.randn(total, heads * group, head_dim, generator=g).bfloat16(), R(total), R(total)] for _ in range(2)]
        for l in range(2):
            for dst, src in zip((q[l], k[l], v[l]), new[l]):
                dst[:total] = src.to(DEV)
                dst[total:] = float("nan")
        n_new.copy_(i32(counts))
        keep.copy_(i32([a + b for a, b in zip(lens, accepted)]))
        if graph is not None:
            graph.replay()
        else:
            outs = s.decode(q, k, v, n_new, tokens, most)
            quant.table_trim(s.text, keep)
        starts = [0]
        for c in counts:
            starts.append(starts[-1] + c)
        for l in range(2):
            full = [[torch.cat([kept[l][i][b], new[l][1 + i][starts[b]:starts[b + 1]]]) for b in range(seqs)] for i in range(2)]
            check_attend(outs[l][0], outs[l][1], starts, None, [lens[b] + counts[b] for b in range(seqs)], new[l][0], [held(x) for x in full[0]],
                         [held(x) for x in full[1]], group, head_dim ** -0.5, visual=(new[0][0], vis_held[0][0], vis_held[l][1]))
            for i in range(2):
                kept[l][i] = [full[i][b][: lens[b] + accepted[b]] for b in range(seqs)]
        lens = [a + b for a, b in zip(lens, accepted)]
        assert s.text.lens.tolist() == lens
    s.text.check(), s.visual.check()
    for table in (s.text, s.visual):
        quant.table_trim(table)
        assert int(table.state[0]) == table.free.numel() and sorted(table.free.tolist()) == list(range(table.free.numel()))


def test_two_calls_at_once_on_two_streams_and_the_same_again():
    c = Cache([900, 35, 1300, 4], 4, 128, 16, 2)
    starts, q = queries([1] * 4, 8, 128, 1)
    qd = q.to(DEV)
    want = quant.attend(c.stream(qd), 4, 16, seq_ids=c.ids)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(20):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(quant.attend(c.stream(qd), 4, 16, seq_ids=c.ids))
    torch.cuda.synchronize()
    for out, lse in got:       # sums are taken in one order: the same bits
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    check_attend(*want, starts, None, c.lens, q, c.k_held, c.v_held, 2, 128 ** -0.5)
