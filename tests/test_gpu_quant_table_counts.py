"""Counts of a table call that lie in the table itself (every sequence doubled, halves of another's length kept): all of them are read
before any of the table is written."""

import random

import pytest
import torch

from oracle import quant_cache as O
from paper_2602_01901_b200 import quant

from test_gpu_quant_attend import i32
from test_gpu_quant_cache import same_table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,most,room", [(7, 60, 600), (900, 40, 3600), (4000, 3, 9000), (300, 90, 40000)], ids=str)
@pytest.mark.parametrize("listed", [False, True], ids=["in_order", "listed"])
def test_as_many_new_tokens_as_a_row_has(seqs, most, room, listed):
    rng, page = random.Random(seqs), 16
    per = -(-3 * most // page)
    table, model = quant.PageTable.empty(seqs, per, page, seqs * per), O.Table(seqs, per, page, seqs * per)
    lens = [rng.randint(0, most) for _ in range(seqs)]
    quant.table_extend(table, i32(lens), max_slots=sum(lens))
    model.extend(range(seqs), lens, sum(lens))
    ids = rng.sample(range(seqs), seqs) if listed else list(range(seqs))
    counts = list(model.lens)          # the i-th of the list takes what row i has
    room = max(room, sum(counts))
    want = model.extend(ids, counts, room)
    starts, slots = quant.table_extend(table, table.lens, seq_ids=i32(ids) if listed else None, max_slots=room)
    assert (starts.tolist(), slots.tolist()) == want
    same_table(table, model)
    model.trim(ids, list(model.lens))      # and the i-th of the list keeps as many as row i has
    quant.table_trim(table, table.lens, seq_ids=i32(ids) if listed else None)
    same_table(table, model)
