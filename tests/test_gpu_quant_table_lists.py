"""Page tables in calls that list thousands of sequences: every list up to the documented most, as the first long call of a
process (what a longer call before it sets for the kernel would hide what a shorter one needs)."""

import os
import subprocess
import sys

import pytest
import torch

from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

# A call holds 16 bytes a sequence in shared memory, and a bit for every row of the table where ids are given; 48 KB is what a
# kernel has without being given more, its own variables among them.
LISTS = {
    "without_ids": (4096, False, [2048, 3000, 3039, 3040, 3041, 3056, 3071, 3073, 4096]),
    "ids_of_4096_rows": (4096, True, [2500, 3007, 3008, 3039, 3040, 3041, 4096]),
    "ids_of_65536_rows": (qc.QC_TABLE_MAX_SEQS, True, [2048, 2527, 2528, 2544, 2560, 2561, 4096]),
}


def run(rows, listed, sizes, first):
    """Each size: a token each, a second one each, down to one, released.  `first`: the call that is made before the others."""
    page = 16
    for n in sizes:
        table = quant.PageTable.empty(rows, 2, page, n + 5)
        ids = torch.randperm(rows, generator=torch.Generator().manual_seed(n))[:n] if listed else torch.arange(n)
        given = ids.to(torch.int32).cuda() if listed else None
        ones = torch.ones(n, dtype=torch.int32, device="cuda")
        if first == "trim":
            quant.table_trim(table, ones, seq_ids=given)
            quant.table_trim(table, seq_ids=given, n_seqs=None if listed else n)
        for position in range(2):
            starts, slots = quant.table_extend(table, seq_ids=given, n_seqs=None if listed else n)
            assert torch.equal(starts.cpu(), torch.arange(n + 1, dtype=torch.int32)), n
            assert torch.equal(slots.cpu(), torch.arange(n, dtype=torch.int32) * page + position), n
            assert torch.equal(table.lens.cpu()[ids], torch.full((n,), position + 1, dtype=torch.int32)), n
            assert torch.equal(table.pages.cpu()[ids, 0], torch.arange(n, dtype=torch.int32)) and int(table.state[0]) == 5, n
        quant.table_trim(table, ones, seq_ids=given)
        assert torch.equal(table.lens.cpu()[ids], ones.cpu()) and int(table.lens.sum()) == n and int(table.state[0]) == 5, n
        quant.table_trim(table, seq_ids=given, n_seqs=None if listed else n)
        assert int(table.lens.sum()) == 0 and bool((table.pages == -1).all()) and int(table.state[0]) == n + 5, n
        assert torch.equal(table.free.cpu(), torch.arange(n + 4, -1, -1, dtype=torch.int32)), n
        table.check()


@pytest.mark.parametrize("first", ["extend", "trim"])
@pytest.mark.parametrize("kind", list(LISTS))
def test_lists_of_every_length_in_a_process_of_their_own(kind, first):
    code = f"import sys; sys.path[:0] = {[HERE, os.path.dirname(HERE)]!r}\nimport test_gpu_quant_table_lists as t\nt.run(*t.LISTS[{kind!r}], {first!r})"
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
