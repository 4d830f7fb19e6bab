"""Rotations of the oracle against hand-made numbers, and what the calls on positions and bf16 pages refuse on the host (no GPU needed)."""

import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import positions as O
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import build as qbuild
from paper_2602_01901_b200 import paged


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return qc.load()


def status_of(call):
    try:
        call()
    except qc.QcError as e:
        return e.status
    return qc.QC_OK


def test_a_rotation_by_hand():
    x = [[[1.0, 2.0, 3.0, 4.0, 5.0]]]
    quarter = math.pi / 2
    assert np.allclose(O.turned(x, [[1], [2]], [quarter, quarter], [0, 1], False), [[[-3.0, -2.0, 1.0, -4.0, 5.0]]])
    assert np.allclose(O.turned(x, [[1], [2]], [quarter, quarter], [0, 1], True), [[[-2.0, 1.0, -3.0, -4.0, 5.0]]])
    assert np.allclose(O.normed([3.0, 4.0], [1.0, 2.0], 0.0), [3 / math.sqrt(12.5), 8 / math.sqrt(12.5)])


@pytest.mark.parametrize("adjacent", [False, True])
def test_a_rotation_keeps_lengths_and_differences_of_positions(adjacent):
    rng = np.random.default_rng(3)
    a, b, freqs = rng.normal(size=(1, 1, 16)), rng.normal(size=(1, 1, 16)), rng.uniform(0.01, 1.0, 6)
    turn = lambda x, p: O.turned(x, [[p]], freqs, [0] * 6, adjacent)
    assert np.isclose(np.linalg.norm(turn(a, 7)), np.linalg.norm(a))
    assert np.isclose((turn(a, 107) * turn(b, 103)).sum(), (turn(a, 4) * turn(b, 0)).sum())


# ---- refusals of the C calls: none of them touches a device -------------------------------------------------

NO_DEVICE = 4096      # one that is not there: a call that passes the checks ends at it
BIG = 1 << 20
ROWS = dict(n_tokens=2, n_q_heads=4, n_kv_heads=2, head_dim=128, rotary_dim=128, n_axes=1, freqs_dev=64, positions_dev=64, eps=1e-6,
            q_dev=BIG, q_stride=512, q_out_dev=2 * BIG, q_out_stride=512, k_dev=3 * BIG, k_stride=256, k_out_dev=4 * BIG, k_out_stride=256)

BAD_ROWS = [
    (dict(head_dim=96), 2), (dict(head_dim=0), 2), (dict(n_tokens=-1), 1), (dict(n_tokens=qc.QC_PAGED_MAX_TOKENS + 1), 2), (dict(n_q_heads=0), 1), (dict(n_q_heads=-1), 1),
    (dict(n_kv_heads=0), 1), (dict(n_q_heads=qc.QC_PAGED_MAX_HEADS + 1), 2), (dict(n_kv_heads=qc.QC_PAGED_MAX_HEADS + 1), 2),
    (dict(rotary_dim=24), 1), (dict(rotary_dim=-16), 1), (dict(rotary_dim=144), 1), (dict(n_axes=0), 1), (dict(n_axes=qc.QC_ROTATE_MAX_AXES + 1), 2),
    (dict(n_axes=2, position_stride=-1), 1), (dict(freqs_dev=0), 1), (dict(freqs_dev=66), 1), (dict(axes_dev=66), 1), (dict(positions_dev=0), 1), (dict(positions_dev=65), 1),
    (dict(q_norm_dev=72), 1), (dict(k_norm_dev=72), 1), (dict(eps=-1.0), 1), (dict(eps=math.nan), 1), (dict(eps=math.inf), 1),
    (dict(q_dev=BIG + 8), 1), (dict(q_dev=0), 1), (dict(q_out_dev=0), 1), (dict(q_out_dev=2 * BIG + 8), 1), (dict(q_stride=-8), 1), (dict(q_stride=516), 1),
    (dict(q_out_stride=504), 1), (dict(k_dev=3 * BIG + 2), 1), (dict(k_stride=-8), 1), (dict(k_stride=257), 1),
]


@pytest.mark.parametrize("change,status", BAD_ROWS + [
    (dict(k_dev=0), 1), (dict(k_out_dev=0), 1), (dict(k_out_stride=248), 1), (dict(q_dev=0, q_out_dev=0, k_dev=0, k_out_dev=0), 1),
    (dict(q_out_dev=BIG + 16), 1), (dict(q_out_dev=BIG, q_stride=1024), 1), (dict(q_out_dev=3 * BIG), 1), (dict(k_out_dev=BIG), 1), (dict(k_out_dev=2 * BIG + 1024), 1),
])
def test_rows_that_are_none_are_refused(change, status):
    assert status_of(lambda: qc.qc_rotate(NO_DEVICE, 0, qc.qc_rotate_args(**{**ROWS, **change}))) == status


APPEND = dict(v_dev=5 * BIG, v_stride=256, slots_dev=64, page_size=16, n_pages=4, k_pool_dev=6 * BIG, v_pool_dev=7 * BIG)


def append_args(rows=None, **change):
    return qc.qc_paged_append_args(rows=qc.qc_rotate_args(**{**ROWS, "k_out_dev": 0, "k_out_stride": 0, **(rows or {})}), **{**APPEND, **change})


@pytest.mark.parametrize("change,status", [(dict(rows=c), s) for c, s in BAD_ROWS] + [
    (dict(page_size=8), 2), (dict(page_size=0), 2), (dict(n_pages=0), 1), (dict(n_pages=1 << 27), 2), (dict(rows=dict(k_dev=0)), 1), (dict(k_pool_dev=0), 1), (dict(v_pool_dev=0), 1),
    (dict(v_dev=0), 1), (dict(rows=dict(k_dev=0), v_dev=0, k_pool_dev=0, v_pool_dev=0), 1), (dict(rows=dict(k_out_dev=4 * BIG)), 1), (dict(slots_dev=0), 1), (dict(slots_dev=66), 1),
    (dict(v_stride=-8), 1), (dict(v_stride=260), 1), (dict(v_dev=5 * BIG + 8), 1), (dict(k_pool_dev=6 * BIG + 8), 1), (dict(v_pool_dev=7 * BIG + 2), 1),
    (dict(v_pool_dev=6 * BIG), 1), (dict(k_pool_dev=3 * BIG), 1), (dict(v_pool_dev=5 * BIG + 256), 1), (dict(k_pool_dev=BIG + 512), 1),
    (dict(rows=dict(q_out_dev=6 * BIG + 1024)), 1), (dict(rows=dict(q_out_dev=5 * BIG)), 1), (dict(rows=dict(k_out_dev=0, k_out_stride=0, q_out_dev=3 * BIG)), 1),
])
def test_an_append_that_is_none_is_refused(change, status):
    assert status_of(lambda: qc.qc_paged_append(NO_DEVICE, 0, append_args(**change))) == status


# q, k and v as parts of one fused tensor of 2 tokens: 4 + 2 + 2 heads
FUSED = dict(q_dev=BIG, q_stride=1024, k_dev=BIG + 1024, k_stride=1024)


@pytest.mark.parametrize("rows,fine", [
    (dict(**FUSED, q_out_dev=BIG, q_out_stride=1024), True), (dict(**FUSED, q_out_dev=BIG, q_out_stride=512), False),
    (dict(**FUSED, q_out_dev=BIG + 512, q_out_stride=1024), False), (dict(**FUSED, q_out_dev=BIG + 1536, q_out_stride=1024), False),
    (dict(**FUSED, q_out_dev=BIG - 2048, q_out_stride=512), True), (dict(**FUSED, q_out_dev=BIG - 2032, q_out_stride=512), False),
    (dict(**FUSED, q_out_dev=BIG + 3584, q_out_stride=512), False), (dict(**FUSED, q_out_dev=BIG + 4096, q_out_stride=512), True),
])
def test_an_output_may_lie_over_its_own_rows_and_no_others(rows, fine):
    call = lambda: qc.qc_paged_append(NO_DEVICE, 0, append_args(rows=rows, v_dev=BIG + 1536, v_stride=1024))
    assert status_of(call) == (qc.QC_ERR_CUDA if fine else qc.QC_ERR_INVALID_ARG)


def test_no_tokens_and_null_pointers(lib):
    assert status_of(lambda: qc.qc_rotate(NO_DEVICE, 0, qc.qc_rotate_args(**{**ROWS, "n_tokens": 0}))) == qc.QC_OK
    assert status_of(lambda: qc.qc_paged_append(NO_DEVICE, 0, append_args(rows=dict(n_tokens=0), slots_dev=0))) == qc.QC_OK
    assert lib.qc_rotate(0, None, None) == lib.qc_paged_append(0, None, None) == qc.QC_ERR_INVALID_ARG


def test_a_good_call_without_its_device_is_an_error_status():
    assert status_of(lambda: qc.qc_rotate(NO_DEVICE, 0, qc.qc_rotate_args(**ROWS))) == qc.QC_ERR_CUDA
    assert status_of(lambda: qc.qc_paged_append(NO_DEVICE, 0, append_args())) == qc.QC_ERR_CUDA


def test_host_tensors_are_refused():
    x, slots, pool = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16)
    for call in (lambda: paged.rotate(x, x, slots, paged.Rotation(torch.ones(32))), lambda: paged.append(pool, pool, slots, x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for call in (lambda: paged.rotate(None, None, slots, None), lambda: paged.append(None, None, slots, None, None), lambda: paged.append(pool, None, slots, None, x),
                 lambda: paged.rotate(None, x, slots, None, q_out=x), lambda: paged.rotate([1], x, slots, None)):
        with pytest.raises(ValueError):
            call()


# ---- attention ----------------------------------------------------------------------------------------------

STREAM = dict(q_dev=BIG, q_stride=512, k_pool_dev=64, v_pool_dev=64, pages_dev=64, lens_dev=64, max_pages=4, n_pages=9, rows=3)


def attend_args(own=None, shared=None, **change):
    a = qc.qc_paged_attend_args(n_q_heads=4, n_kv_heads=2, head_dim=128, page_size=16, n_seqs=2, n_tokens=2, max_queries=1, causal=1, out_dev=2 * BIG, workspace_dev=256,
                                workspace_bytes=1 << 40, own=qc.qc_paged_stream(**{**STREAM, **(own or {})}))
    if shared is not None:
        a.shared, a.n_groups = qc.qc_paged_stream(**{**STREAM, **shared}), 1
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=80), 2), (dict(page_size=48), 2), (dict(n_q_heads=5), 1), (dict(n_q_heads=0), 1), (dict(n_kv_heads=0), 1), (dict(n_seqs=0), 1), (dict(n_seqs=4, n_tokens=4), 1),
    (dict(n_tokens=-1), 1), (dict(n_tokens=1), 1), (dict(n_tokens=qc.QC_PAGED_MAX_TOKENS + 1), 2), (dict(max_queries=0), 1), (dict(max_queries=qc.QC_PAGED_MAX_QUERIES + 1), 2),
    (dict(n_seqs=qc.QC_PAGED_MAX_SEQS + 1, seq_ids_dev=64), 2), (dict(n_q_heads=2 * qc.QC_PAGED_MAX_HEADS), 2), (dict(own=dict(q_dev=0)), 1), (dict(out_dev=0), 1), (dict(out_dev=2 * BIG + 8), 1),
    (dict(lse_out_dev=66), 1), (dict(status_dev=65), 1), (dict(seq_ids_dev=66), 1), (dict(starts_dev=66), 1), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=math.nan), 1),
    (dict(softmax_scale=math.inf), 1), (dict(workspace_dev=264), 1), (dict(workspace_dev=0), 1), (dict(workspace_bytes=8), 1), (dict(out_dev=BIG), 1), (dict(out_dev=BIG + 2032), 1), (dict(out_dev=BIG - 1024), 1),
    (dict(own=dict(q_dev=BIG + 8)), 1), (dict(own=dict(q_stride=-8)), 1), (dict(own=dict(q_stride=12)), 1), (dict(own=dict(k_pool_dev=0)), 1), (dict(own=dict(v_pool_dev=24)), 1),
    (dict(own=dict(pages_dev=0)), 1), (dict(own=dict(lens_dev=62)), 1), (dict(own=dict(max_pages=0)), 1), (dict(own=dict(n_pages=0)), 1), (dict(own=dict(rows=0)), 1),
    (dict(own=dict(max_pages=1 << 27)), 2), (dict(own=dict(n_pages=1 << 27)), 2), (dict(own=dict(n_pages=1 << 26)), 2),
    (dict(n_groups=1), 1), (dict(groups_dev=64), 1), (dict(shared_ids_dev=64), 1), (dict(shared=dict(q_dev=0)), 1), (dict(shared=dict(rows=0)), 1), (dict(shared={}, n_groups=2), 1),
    (dict(shared={}, n_groups=-1), 1), (dict(shared={}, n_groups=4, groups_dev=64), 1), (dict(shared={}, n_groups=qc.QC_PAGED_MAX_SEQS + 1, groups_dev=64, shared_ids_dev=64), 2),
    (dict(shared=dict(q_dev=2 * BIG + 1024)), 1), (dict(shared=dict(n_pages=1 << 28)), 2), (dict(shared={}, groups_dev=66), 1), (dict(shared={}, shared_ids_dev=66), 1),
])
def test_attention_refuses_what_it_can_see_on_the_host(change, status):
    assert status_of(lambda: qc.qc_paged_attend(NO_DEVICE, 0, attend_args(**change))) == status


FAR = 3 * BIG


@pytest.mark.parametrize("change", [
    dict(own=dict(k_pool_dev=FAR)), dict(own=dict(v_pool_dev=FAR - 2 * 9 * 16 * 128 * 2 + 16)), dict(own=dict(pages_dev=FAR + 28)), dict(own=dict(lens_dev=FAR - 8)), dict(seq_ids_dev=FAR - 4),
    dict(starts_dev=FAR - 8), dict(status_dev=FAR + 4), dict(shared=dict(k_pool_dev=FAR + 16)), dict(shared={}, groups_dev=FAR - 4), dict(shared={}, shared_ids_dev=FAR),
    dict(shared=dict(q_dev=FAR - 1024)),
])
def test_attention_writes_over_nothing_that_it_reads(change):
    """Rows written (2048 bytes here), or their sums of exponentials (32), against every other argument."""
    for mine in (dict(out_dev=FAR), dict(lse_out_dev=FAR)):
        assert status_of(lambda: qc.qc_paged_attend(NO_DEVICE, 0, attend_args(**mine, **change))) == qc.QC_ERR_INVALID_ARG
    assert status_of(lambda: qc.qc_paged_attend(NO_DEVICE, 0, attend_args(out_dev=FAR + BIG, lse_out_dev=FAR + 2 * BIG, **change))) == qc.QC_ERR_CUDA


@pytest.mark.parametrize("at,status", [(FAR - 32, 5), (FAR - 28, 1), (FAR + 2044, 1), (FAR + 2048, 5)])
def test_the_two_outputs_of_attention_lie_apart(at, status):
    assert status_of(lambda: qc.qc_paged_attend(NO_DEVICE, 0, attend_args(out_dev=FAR, lse_out_dev=at))) == status


def test_attention_refuses_a_workspace_that_is_too_small(lib):
    a = attend_args(shared={})
    need = qc.qc_paged_workspace_bytes(a)
    for size, status in ((need - 1, qc.QC_ERR_INVALID_ARG), (need, qc.QC_ERR_CUDA)):
        a.workspace_bytes = size
        assert status_of(lambda: qc.qc_paged_attend(NO_DEVICE, 0, a)) == status
    n = C.c_size_t()
    assert lib.qc_paged_attend(0, None, None) == lib.qc_paged_workspace_bytes(None, C.byref(n)) == lib.qc_paged_workspace_bytes(C.byref(a), None) == qc.QC_ERR_INVALID_ARG


def test_host_tensors_of_streams_are_refused():
    x, ids, pool = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        paged.attend(paged.Stream(x, pool, pool, ids[None], ids))
    with pytest.raises(ValueError, match="Stream"):
        paged.attend((x, pool))
