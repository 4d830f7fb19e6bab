"""Outputs of attention that lie over its queries: each row at its query's place or none at all (no GPU needed)."""

import pytest
import torch

from paper_2602_01901_b200 import binding as qc

from test_quant_cpu import attend_args, lib, status_of      # noqa: F401  (lib: builds the library)

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run")
ROW = 4 * 128 * 2                  # bytes of a token's heads
Q = 1 << 20


def refused(*args, **kw):
    """Whether the call is refused; one that is not finds no device."""
    a = attend_args(stream=dict(q_dev=kw.get("q", Q), q_stride=kw.get("stride", ROW // 2)), visual=kw.get("visual"), n_seqs=1, n_tokens=args[0], out_dev=args[1])
    status = status_of(lambda: qc.qc_quant_attend(0, 0, a))
    assert status in (qc.QC_ERR_INVALID_ARG, qc.QC_ERR_CUDA)
    return status == qc.QC_ERR_INVALID_ARG


@pytest.mark.parametrize("n", [1, 2, 7, 300])
def test_dense_queries(n):
    assert not refused(n, Q)                                       # in place
    assert not refused(n, Q + n * ROW) and not refused(n, Q - n * ROW)
    for off in (16, ROW - 16, ROW, n * ROW - 16):
        if 0 < off < n * ROW:
            assert refused(n, Q + off) and refused(n, Q - off), off


def test_rows_apart():
    s = 5 * ROW // 2                                               # q is the first of five parts of a fused row
    assert refused(3, Q, stride=s) and not refused(1, Q, stride=s)
    assert not refused(1, Q + ROW, stride=s) and refused(2, Q + 4 * ROW, stride=s)
    assert not refused(4, Q + ROW, stride=s) and refused(5, Q + ROW, stride=s)      # four tokens' outputs fit between two queries
    assert not refused(4, Q + 6 * ROW, stride=s) and refused(4, Q + 6 * ROW + 16, stride=s)
    assert refused(3, Q - 16, stride=s) and not refused(3, Q - 3 * ROW, stride=s) and refused(3, Q - 3 * ROW + 16, stride=s)
    assert not refused(3, Q + 2 * 5 * ROW + ROW, stride=s) and refused(3, Q + 2 * 5 * ROW + ROW - 16, stride=s)


def test_one_row_for_all():
    assert refused(3, Q, stride=0) and not refused(1, Q, stride=0)
    assert not refused(3, Q + ROW, stride=0) and refused(3, Q + ROW - 16, stride=0) and refused(3, Q - 3 * ROW + 16, stride=0) and not refused(3, Q - 3 * ROW, stride=0)


def test_the_visual_queries_count_too():
    far = 1 << 30
    assert not refused(4, far, visual=dict(q_dev=far, q_stride=ROW // 2)) and refused(4, far + 16, visual=dict(q_dev=far, q_stride=ROW // 2))
    assert not refused(4, Q, visual=dict(q_dev=Q, q_stride=ROW // 2)) and refused(4, Q, visual=dict(q_dev=Q + ROW, q_stride=ROW // 2))
