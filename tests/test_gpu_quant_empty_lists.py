"""A step without sequences: lists of none are taken by every call of the module and change nothing."""

import pytest
import torch

from paper_2602_01901_b200 import quant

from quant_util import DEV
from test_gpu_quant_attend import i32
from test_gpu_quant_replays import cache

pytestmark = pytest.mark.gpu
NONE = torch.empty(0, dtype=torch.int32)


def test_tables_take_lists_of_none():
    table = quant.PageTable.empty(5, 3, 16, 9)
    quant.table_extend(table, i32([20, 3]), seq_ids=i32([4, 1]), max_slots=23)
    before = [t.clone() for t in (table.pages, table.lens, table.free, table.state)]
    none = NONE.to(DEV)
    for n_new, ids, n_seqs, most in ((none, none, None, 6), (none, None, None, 0), (None, none, None, None), (None, None, 0, None), (none, none, 0, 5000)):
        starts, slots = quant.table_extend(table, n_new, seq_ids=ids, n_seqs=n_seqs, max_slots=most)
        assert starts.dtype == slots.dtype == torch.int32 and starts.tolist() == [0] and slots.tolist() == [-1] * (most or 0)
        quant.table_trim(table, n_new, seq_ids=ids, n_seqs=n_seqs)
    for a, b in zip((table.pages, table.lens, table.free, table.state), before):
        assert torch.equal(a, b)


def test_a_whole_step_of_none_with_padded_tokens():
    s = cache([300, 40], 2, 4, 64, 32, 1)
    none, q = NONE.to(DEV), torch.randn(6, 8, 64, device=DEV).bfloat16()
    for starts in (None, i32([0])):
        out = torch.full_like(q, 9)
        got, lse = quant.attend(s._replace(q=q), 2, 32, seq_ids=none if starts is None else None, starts=starts, max_queries=2, out=out)
        assert got is out and (out == 9).all() and lse.shape == (6, 8)
    slots = torch.full((6,), -1, dtype=torch.int32, device=DEV)
    before = s.k_pool.clone()
    quant.append(s.k_pool, s.v_pool, slots, q[:, :2], q[:, 2:4], 32)
    assert torch.equal(s.k_pool, before)
    with pytest.raises(ValueError):
        quant.attend(s._replace(q=q), 2, 32, seq_ids=none, starts=i32([0, 6]))
