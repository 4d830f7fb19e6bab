"""Page tables on the device, and rows quantised into 4-bit pages and read back, against the integer model and the
row-by-row oracle.  Whole numbers have to be equal, codes and parameters too: the subtraction of two bf16 numbers and the
product with one leave no room for another code except where their exponents are more than 16 apart, which no row here has."""

import math
import random

import numpy as np
import pytest
import torch

from oracle import quant_cache as O
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

from quant_util import DEV, gen, rows

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def same_table(table, model):
    assert int(table.state[1]) == qc.QC_OK
    assert table.lens.tolist() == model.lens
    assert int(table.state[0]) == len(model.free)
    assert table.free[: len(model.free)].tolist() == model.free
    for row, pages in zip(table.pages.tolist(), model.pages):
        assert row == pages + [-1] * (model.max_pages - len(pages))


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("seqs,most", [(1, 70), (5, 200), (300, 90), (1500, 40)])
def test_tables_follow_the_integer_model_through_a_random_run(page, seqs, most):
    rng = random.Random(page * 10000 + seqs)
    max_pages = -(-3 * most // page)
    n_pages = seqs * max_pages * 2 // 3 + 2
    table, model = quant.PageTable.empty(seqs, max_pages, page, n_pages), O.Table(seqs, max_pages, page, n_pages)
    same_table(table, model)
    for step in range(12):
        ids = rng.sample(range(seqs), rng.randint(1, seqs))
        if step % 3 < 2:
            new = [min(rng.choice([0, 1, 1, rng.randint(0, most)]), max_pages * page - model.lens[i]) for i in ids]
            room = sum(new) + rng.randint(0, 9)
            try:
                want = model.extend(ids, new, room)
            except O.Refused:
                want = ([0] * (len(ids) + 1), [-1] * room)
                starts, slots = quant.table_extend(table, i32(new), seq_ids=i32(ids), max_slots=room)
                assert int(table.state[1]) == qc.QC_ERR_OOM_PAGES
                table.state[1] = 0
            else:
                starts, slots = quant.table_extend(table, i32(new), seq_ids=i32(ids), max_slots=room)
            assert starts.tolist() == want[0] and slots.tolist() == want[1]
        else:
            keep = [rng.randint(0, model.lens[i] + 3) for i in ids]
            model.trim(ids, keep)
            quant.table_trim(table, i32(keep), seq_ids=i32(ids))
        same_table(table, model)
    quant.table_trim(table)
    model.trim(list(range(seqs)), [0] * seqs)
    same_table(table, model)
    assert int(table.state[0]) == n_pages


def test_a_table_stays_with_its_tensors():
    table = quant.PageTable.empty(2, 3, 16, 5)
    for name in quant.PageTable.__slots__:
        with pytest.raises(AttributeError):
            setattr(table, name, getattr(table, name))
    table.check()


def test_one_token_each_without_lists_and_slots_of_a_long_call():
    table, model = quant.PageTable.empty(7, 3000, 16, 7 * 3000), O.Table(7, 3000, 16, 7 * 3000)
    for _ in range(18):
        starts, slots = quant.table_extend(table)
        assert (starts.tolist(), slots.tolist()) == model.extend(range(7), [1] * 7, 7)
    long = [9000, 0, 1, 25000, 17, 3, 400]       # more slots than the block that makes the table writes itself
    starts, slots = quant.table_extend(table, i32(long), max_slots=40000)
    assert (starts.tolist(), slots.tolist()) == model.extend(range(7), long, 40000)
    same_table(table, model)


@pytest.mark.parametrize("what,status", [("id", 1), ("negative_id", 1), ("negative_count", 1), ("twice", 4), ("pages", 3), ("row", 3), ("slots", 1)])
@pytest.mark.parametrize("long", [False, True], ids=["short", "long"])
def test_what_cannot_be_done_as_a_whole_changes_nothing(what, status, long):
    table = quant.PageTable.empty(6, 700, 16, 900)
    model = O.Table(6, 700, 16, 900)
    quant.table_extend(table, i32([20, 3, 600]), seq_ids=i32([4, 0, 1]), max_slots=623)
    model.extend([4, 0, 1], [20, 3, 600], 623)
    ids, new, room = [2, 4, 0], [5, 40, 1], 9000 if long else 60
    if what == "id":
        ids[1] = 6
    elif what == "negative_id":
        ids[2] = -1
    elif what == "negative_count":
        new[0] = -1
    elif what == "twice":
        ids[2] = 2
    elif what == "pages":
        new[:2], room = [7000, 7000], 20000 if long else 8000
        new[1] = 7000
    elif what == "row":
        new[0], room = 700 * 16 + 1, 20000 if long else 8000
    elif what == "slots":
        room = 45 if not long else 8300
        new = [5, 40, 1] if not long else [5, 4000, 4300]
    starts, slots = quant.table_extend(table, i32(new), seq_ids=i32(ids), max_slots=room)
    assert int(table.state[1]) == status
    with pytest.raises(qc.QcError) as e:
        table.check()
    assert e.value.status == status
    assert starts.tolist() == [0] * 4 and slots.tolist() == [-1] * room
    table.state[1] = 0
    same_table(table, model)
    if what in ("id", "negative_id", "negative_count", "twice"):
        quant.table_trim(table, i32(new), seq_ids=i32(ids))
        assert int(table.state[1]) == status
        table.state[1] = 0
        same_table(table, model)


# ---- rows ------------------------------------------------------------------------------------------

def pools(heads, head_dim, page, n_pages):
    made = [quant.empty_pool(heads, head_dim, page, n_pages) for _ in "kv"]
    for p in made:
        p.fill_(0xA5)
    return made


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads,tokens,layout", [(1, 1, "scattered"), (3, 37, "scattered"), (4, 60, "run"), (9, 21, "run"), (2, 700, "runs"), (8, 530, "run")])
def test_rows_are_held_as_the_format_says_and_nothing_else_is_touched(page, head_dim, heads, tokens, layout):
    g = gen(tokens * 7 + heads + page + head_dim)
    n_pages = tokens + 2 if layout == "scattered" else -(-tokens // page) + 9
    fused = rows(tokens, 3 * heads + 1, head_dim, g)
    k, v = fused[:, heads:2 * heads], fused[:, 2 * heads:3 * heads]                 # strided, as a fused projection's output
    if layout == "scattered":
        slots = torch.randperm(n_pages, generator=g)[:tokens] * page + torch.randint(0, page, (tokens,), generator=g)
    else:
        order = torch.randperm(n_pages, generator=g)
        i = torch.arange(tokens) + 5
        if layout == "runs":       # several sequences: runs begin anywhere and skip
            i = i + (torch.arange(tokens) // 53) * 7
        i = i[i // page < n_pages]
        slots = order[i // page] * page + i % page
        slots = torch.cat([slots, torch.full((tokens - len(slots),), -1)])
    slots[torch.randperm(tokens, generator=g)[: tokens // 9]] = -1                  # holes: padded tokens
    if tokens > 3:
        slots[1] = n_pages * page                                                     # behind the pool
    k_pool, v_pool = pools(heads, head_dim, page, n_pages)
    before = k_pool.cpu().numpy().copy()
    d = lambda t: t.to(DEV)
    fused_d = d(fused)
    quant.append(k_pool, v_pool, d(slots.to(torch.int32)), fused_d[:, heads:2 * heads], fused_d[:, 2 * heads:3 * heads], page)
    got = {"k": k_pool.cpu().numpy(), "v": v_pool.cpu().numpy()}
    n_codes = heads * page * head_dim // 2
    picked = range(tokens) if tokens < 80 else sorted(random.Random(1).sample(range(tokens), 60)) + list(range(tokens - 6, tokens))
    live = [t for t in range(tokens) if 0 <= int(slots[t]) < n_pages * page]
    for which, x in (("k", k), ("v", v)):
        a = x.double().numpy()
        for t in picked:
            if t not in live:
                continue
            for h in range(heads):
                lo, r, codes = O.row_at(got[which], which, heads, head_dim, page, int(slots[t]), h)
                lo0, r0, codes0 = O.quantise(a[t, h])
                assert (lo, r) == (lo0, r0) and np.array_equal(codes, codes0), (which, t, h)
        # bytes of rows that nobody stored are what they were
        touched = np.zeros(before.shape, bool)
        places = {}
        for t in live:
            s = int(slots[t])
            for h in range(heads):
                key = (s % page, h)
                if key not in places:
                    places[key] = sorted({O.code_place(which, head_dim, h, page, s % page, e)[0] for e in range(0, head_dim, 2)})
                touched[s // page, places[key]] = True
                at = n_codes + (h * page + s % page) * 4
                touched[s // page, at:at + 4] = True
        assert np.array_equal(got[which][~touched], before[~touched])
        if len(live) == len(set(int(slots[t]) for t in live)) and tokens > 1:
            assert touched.sum() == len(live) * heads * (head_dim // 2 + 4)
    # and back: the nearest bf16 to what the row stands for, whose sum in fp32 may fall to the other side of a tie
    back_k, back_v = quant.read(k_pool, v_pool, d(slots.to(torch.int32)), heads, head_dim, page)
    for back, x in ((back_k, k), (back_v, v)):
        b, a = back.double().cpu().numpy(), x.double().numpy()
        for t in picked:
            for h in range(heads):
                if t not in live:
                    assert not b[t, h].any()
                    continue
                lo, r, codes = O.quantise(a[t, h])
                exact = O.value(lo, r, codes)
                size = np.abs(exact) + 2.0 ** -14 * (abs(lo) + 15 / r if r else abs(lo))
                assert np.all(np.abs(b[t, h] - exact) <= 2.0 ** -8 * size)
                if r:      # half a step, and the part of a step that r's rounding moves the largest element by
                    assert np.all(np.abs(exact - a[t, h]) <= (0.5 + 15 * 2.0 ** -8) / r)


@pytest.mark.parametrize("head_dim", [64, 128])
def test_rows_at_the_edges_of_the_numbers(head_dim):
    x = torch.zeros(12, 1, head_dim)
    x[0] = 3.25                                        # no range
    x[1, 0, 5] = 2.0 ** -110                           # a range below the least
    x[2, 0, :2] = torch.tensor([-(2.0 ** -100), 2.0 ** -99])
    x[3, 0, 7] = float("nan")
    x[4, 0, 0] = float("inf")
    x[5, 0, -1] = float("-inf")
    x[6, 0, :2] = torch.tensor([3.0e38, -3.0e38])      # a range that is not finite
    x[7, 0, :2] = torch.tensor([1.5e38, -1.5e38])
    x[8] = -torch.arange(head_dim).float()
    x[9, 0, 3] = 1.0                                   # one outlier
    x[10, 0] = torch.linspace(-7.5, 7.5, head_dim)     # ties between codes
    x[11] = -0.0
    x = x.bfloat16()
    k_pool, v_pool = pools(1, head_dim, 16, 1)
    slots = torch.arange(12, dtype=torch.int32, device=DEV)
    quant.append(k_pool, v_pool, slots, x.to(DEV), x.to(DEV), 16)
    for which, pool in (("k", k_pool), ("v", v_pool)):
        raw = pool.cpu().numpy()
        for t in range(12):
            lo, r, codes = O.row_at(raw, which, 1, head_dim, 16, t, 0)
            lo0, r0, codes0 = O.quantise(x[t, 0].double().numpy())
            assert (math.isnan(lo) and math.isnan(lo0) or lo == lo0) and r == r0 and np.array_equal(codes, codes0), (which, t)
    back, _ = quant.read(k_pool, None, slots, 1, head_dim, 16)
    nan = torch.isnan(back).all(-1)[:, 0].tolist()
    assert nan == [t in (3, 4, 5, 6) for t in range(12)]


def test_one_tensor_alone_strides_and_rows_that_stay():
    g = gen(3)
    x = rows(10, 2, 128, g).to(DEV)
    k_pool, v_pool = pools(2, 128, 32, 3)
    before = v_pool.clone()
    slots = torch.tensor([40, 41, -1, 43, 7, 6, 95, 96, -5, 0], dtype=torch.int32, device=DEV)
    quant.append(k_pool, None, slots, x, None, 32)
    assert torch.equal(v_pool, before)
    out = torch.full((10, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    got, none = quant.read(k_pool, None, slots, 2, 128, 32, k_out=out)
    assert none is None and got is out
    for t, s in enumerate(slots.tolist()):
        assert (out[t] == 7.0).all() == (not 0 <= s < 96), t
    # one row for all tokens (a stride of nothing)
    quant.append(None, v_pool, slots[:4], None, x[:1].expand(4, 2, 128), 32)
    _, same = quant.read(None, v_pool, slots[[0, 1, 3]], 2, 128, 32)
    assert torch.equal(same[0], same[1]) and torch.equal(same[0], same[2])


def test_places_behind_four_gigabytes():
    heads, head_dim, page = 32, 128, 64
    n_pages = (5 << 30) // O.page_bytes(heads, head_dim, page)
    k_pool = quant.empty_pool(heads, head_dim, page, n_pages)
    x = rows(6, heads, head_dim, gen(9))
    slots = torch.tensor([n_pages * page - 1 - i * 70 for i in range(6)], dtype=torch.int32, device=DEV)
    quant.append(k_pool, None, slots, x.to(DEV), None, page)
    back, _ = quant.read(k_pool, None, slots, heads, head_dim, page)
    for t in range(6):
        raw = k_pool[int(slots[t]) // page].cpu().numpy()[None]
        lo, r, codes = O.row_at(raw, "k", heads, head_dim, page, int(slots[t]) % page, 31)
        lo0, r0, codes0 = O.quantise(x[t, 31].double().numpy())
        assert (lo, r) == (lo0, r0) and np.array_equal(codes, codes0)
        exact = O.value(lo, r, codes)
        assert np.all(np.abs(back[t, 31].double().cpu().numpy() - exact) <= 2.0 ** -8 * (np.abs(exact) + 2.0 ** -14 * (abs(lo) + 15 / r)))
