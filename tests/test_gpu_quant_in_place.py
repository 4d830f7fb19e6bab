"""Attention whose output takes the place of its queries: the bits of an output elsewhere."""

import pytest
import torch

from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

from test_gpu_quant_replays import cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,kv_heads,group,head_dim", [([30000], 1, 1, 128), ([9001, 50, 7333], 2, 4, 64), ([1900] * 30, 8, 1, 128), ([6000, 9000], 2, 16, 128), ([20] * 70, 2, 2, 64)],
                         ids=["one", "cut", "even", "sixteen", "short"])
@pytest.mark.parametrize("streams", ["text", "both", "visual"])
def test_an_output_in_its_queries_place(lens, kv_heads, group, head_dim, streams):
    text, visual = cache(lens, kv_heads, group, head_dim, 32, 1), cache(lens[::-1], kv_heads, group, head_dim, 32, 2)
    for turn in range(10):
        t, v = (s._replace(q=s.q.clone()) for s in (text, visual))
        if streams == "both":
            v = v._replace(q=t.q)
        second = None if streams == "text" else v
        want, want_lse = quant.attend(t, kv_heads, 32, visual=second)
        place = v.q if streams == "visual" else t.q
        got, lse = quant.attend(t, kv_heads, 32, visual=second, out=place)
        assert got is place and torch.equal(got, want) and torch.equal(lse, want_lse), turn


def test_an_output_over_other_queries_is_refused():
    s = cache([300, 40, 50], 1, 4, 64, 32, 1)
    both = torch.cat([s.q, s.q])
    before = both.clone()
    for stream, out in ((s._replace(q=both[:3]), both[1:4]), (s._replace(q=both[1:4]), both[:3]), (s._replace(q=both[::2]), both[:3])):
        with pytest.raises(qc.QcError) as e:
            quant.attend(stream, 1, 32, out=out)
        assert e.value.status == qc.QC_ERR_INVALID_ARG
    assert torch.equal(both, before)
    quant.attend(s._replace(q=both[:3]), 1, 32, out=both[3:])
    assert torch.equal(both[:3], before[:3]) and not torch.equal(both[3:], before[3:])
