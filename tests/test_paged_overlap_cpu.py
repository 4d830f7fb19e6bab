"""Rows and pools that a call on positions writes, over what it reads besides rows (no GPU needed)."""

import pytest

from paper_2602_01901_b200 import binding as qc

from test_paged_cpu import BIG, NO_DEVICE, ROWS, append_args, lib, status_of      # noqa: F401  (lib: builds the library)

FAR = 16 * BIG
ROW = 2048                         # bytes of two tokens of 4 heads of 128, dense
# what a call reads: its argument, how many bytes of it (2 tokens, 64 pairs, 128 weights)
READ = [(dict(freqs_dev=FAR), 256), (dict(axes_dev=FAR), 256), (dict(positions_dev=FAR), 8), (dict(q_norm_dev=FAR), 256), (dict(k_norm_dev=FAR), 256),
        (dict(q_norm_dev=FAR, norm_f32=1), 512), (dict(k_norm_dev=FAR, norm_f32=1), 512)]


def rotate(**rows):
    return status_of(lambda: qc.qc_rotate(NO_DEVICE, 0, qc.qc_rotate_args(**{**ROWS, **rows})))


@pytest.mark.parametrize("read,size", READ)
@pytest.mark.parametrize("out,written", [("q_out_dev", ROW), ("k_out_dev", ROW // 2)])
def test_rows_lie_over_nothing_else_that_is_read(read, size, out, written):
    for at in (FAR, FAR - written + 16, FAR + (size - 1) // 16 * 16):
        assert rotate(**read, **{out: at}) == qc.QC_ERR_INVALID_ARG, at - FAR
    for at in (FAR - written, FAR + -(-size // 16) * 16):
        assert rotate(**read, **{out: at}) == qc.QC_ERR_CUDA, at - FAR


def test_every_axis_of_the_positions_counts_and_what_lies_between_does_not():
    read = dict(n_axes=3, positions_dev=FAR, position_stride=2048)          # axes 8192 bytes apart
    for axis in range(3):
        assert rotate(**read, q_out_dev=FAR + axis * 8192 - 1024) == qc.QC_ERR_INVALID_ARG
    for at in (FAR + 16, FAR + 8192 - ROW, FAR + 8192 + 16, FAR + 2 * 8192 + 16):
        assert rotate(**read, q_out_dev=at) == qc.QC_ERR_CUDA
    assert rotate(positions_dev=FAR, position_stride=2048, q_out_dev=FAR + 8192 - 1024) == qc.QC_ERR_CUDA      # one axis: no stride


def test_what_a_call_does_not_read_may_be_anywhere():
    assert rotate(rotary_dim=0, freqs_dev=2 * BIG, axes_dev=2 * BIG, positions_dev=2 * BIG) == qc.QC_ERR_CUDA
    assert rotate(k_dev=0, k_out_dev=0, k_norm_dev=2 * BIG) == rotate(q_dev=0, q_out_dev=0, q_norm_dev=4 * BIG) == qc.QC_ERR_CUDA


@pytest.mark.parametrize("read,size", READ + [(None, 8)])
def test_pools_and_queries_of_an_append_lie_over_nothing_else_that_is_read(read, size):
    """Pools are 4 pages of 16 tokens of 2 heads: 32 768 bytes."""
    args = lambda **change: append_args(rows={**(read or {}), **change.pop("rows", {})}, **({} if read else dict(slots_dev=FAR)), **change)
    call = lambda **change: status_of(lambda: qc.qc_paged_append(NO_DEVICE, 0, args(**change)))
    for pool in ("k_pool_dev", "v_pool_dev"):
        for at in (FAR, FAR - 32768 + 16, FAR + (size - 1) // 16 * 16):
            assert call(**{pool: at}) == qc.QC_ERR_INVALID_ARG, (pool, at - FAR)
        for at in (FAR - 32768, FAR + -(-size // 16) * 16):
            assert call(**{pool: at}) == qc.QC_ERR_CUDA, (pool, at - FAR)
    assert call(rows=dict(q_out_dev=FAR - ROW + 16)) == qc.QC_ERR_INVALID_ARG and call(rows=dict(q_out_dev=FAR - ROW)) == qc.QC_ERR_CUDA
