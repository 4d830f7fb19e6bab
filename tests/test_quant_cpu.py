"""The oracle of the 4-bit cache against hand-made numbers, and what the calls refuse on the host (no GPU needed)."""

import ctypes as C
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import quant_cache as O
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import build as qbuild
from paper_2602_01901_b200 import quant


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return qc.load()


def test_bf16_of_the_oracle_rounds_to_nearest_even():
    g = torch.Generator()
    g.manual_seed(1)
    x = torch.cat([torch.randn(500, generator=g) * 2.0 ** torch.randint(-20, 20, (500,), generator=g), torch.arange(1, 64) / 256 + 1])
    assert [O.bf16(float(a)) for a in x] == x.bfloat16().double().tolist()


def test_a_row_by_hand():
    lo, r, codes = O.quantise([0.0, 15.0, 7.0, 7.5, 2.5, 1.5, 0.25])
    assert (lo, r) == (0.0, 1.0) and codes.tolist() == [0, 15, 7, 8, 2, 2, 0]          # ties to even
    lo, r, codes = O.quantise([-1.0, 1.0])
    assert (lo, r) == (-1.0, 7.5) and codes.tolist() == [0, 15] and O.value(lo, r, codes).tolist() == [-1.0, 1.0]
    assert O.quantise([2.0, 2.0])[1] == 0.0 and O.value(2.0, 0.0, [0, 0]).tolist() == [2.0, 2.0]
    assert math.isnan(O.quantise([1.0, math.inf])[0])


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 32)])
def test_every_element_of_a_page_has_a_place_of_its_own(which, head_dim, heads, page):
    places = {O.code_place(which, head_dim, h, page, t, d) for h, t, d in itertools.product(range(heads), range(page), range(head_dim))}
    assert places == set(itertools.product(range(heads * page * head_dim // 2), range(2)))


def test_what_the_lanes_read_is_what_the_format_says():
    """The products take 16 bytes at lane * 16 (and 512 on): for K elements of tokens 2 g and 2 g + 1, for V four tokens' bytes."""
    for lane in range(32):
        g, t = divmod(lane, 4)
        for j in range(32):                  # K, 128 wide: the lane's even token, then (512 on) its odd one
            for odd in range(2):
                assert O.code_place("k", 128, 0, 16, 2 * g + odd, 32 * t + j) == (lane * 16 + j // 2 + 512 * odd, j % 2)
        for j in range(16):
            for odd in range(2):
                assert O.code_place("k", 64, 0, 16, 2 * g + odd, 16 * t + j) == (lane * 16 + j // 2 + 8 * odd, j % 2)
            for i in range(4):
                assert O.code_place("v", 128, 0, 16, 4 * t + i, 16 * g + j) == (j // 8 * 512 + lane * 16 + j // 2 % 4 * 4 + i, j % 2)
        for j in range(8):
            for i in range(4):
                assert O.code_place("v", 64, 0, 16, 4 * t + i, 8 * g + j) == (lane * 16 + j // 2 * 4 + i, j % 2)


def test_the_table_model_takes_and_gives_back_in_order():
    t = O.Table(3, 4, 16, 6)
    assert t.extend([1, 0], [17, 2], 20) == ([0, 17, 19], list(range(16)) + [16, 32, 33, -1])
    t.trim([1, 0], [3, 0])
    assert t.pages == [[], [0], []] and t.free == [5, 4, 3, 2, 1]
    assert t.extend([1, 0], [14, 2], 16)[1] == list(range(3, 16)) + [16, 32, 33]
    for ids, new in (([0, 0], [1, 1]), ([3], [1]), ([0], [-1]), ([2], [100]), ([2], [65])):
        with pytest.raises(O.Refused):
            t.extend(ids, new, 100)


def test_attention_by_hand():
    out, lse = O.attention([1.0, 0.0], [([1.0, 0.0], [[0.0, 5.0], [math.log(3.0), 1.0]], [[0.0, 4.0], [4.0, 0.0]])], 1.0)
    assert np.allclose(out, [3.0, 1.0]) and math.isclose(lse, math.log(4.0))
    assert O.attention([1.0], [([1.0], np.zeros((0, 1)), np.zeros((0, 1)))], 1.0)[1] == -math.inf


def test_many_rows_at_once_are_held_as_one_by_one():
    from quant_util import gen, held, held_torch, rows

    x = rows(200, 2, 64, gen(5))
    a, b = held(x), held_torch(x)
    assert all(np.array_equal(a[name], b[name].numpy()) for name in ("lo", "codes")) and np.allclose(a["step"], b["step"].numpy(), rtol=1e-15)


# ---- refusals of the C calls: none of them touches a device -------------------------------------------

OK_TABLE = dict(max_seqs=4, max_pages=3, page_size=16, n_pages=9, pages_dev=64, lens_dev=64, free_dev=64, state_dev=64)


def status_of(call):
    try:
        call()
    except qc.QcError as e:
        return e.status
    return qc.QC_OK


@pytest.mark.parametrize("change,status", [
    (dict(pages_dev=0), 1), (dict(lens_dev=0), 1), (dict(free_dev=0), 1), (dict(state_dev=0), 1), (dict(state_dev=66), 1), (dict(page_size=24), 2),
    (dict(page_size=0), 2), (dict(max_seqs=0), 1), (dict(max_pages=0), 1), (dict(n_pages=0), 1), (dict(n_pages=-3), 1),
    (dict(max_seqs=qc.QC_TABLE_MAX_SEQS + 1), 2), (dict(n_pages=1 << 27), 2), (dict(max_pages=1 << 27), 2),
])
def test_a_table_that_is_none_is_refused(change, status):
    t = qc.qc_table(**{**OK_TABLE, **change})
    assert status_of(lambda: qc.qc_table_reset(0, 0, t)) == status
    assert status_of(lambda: qc.qc_table_extend(0, 0, t, 1, 0, 0, 1, 64, 64)) == status
    assert status_of(lambda: qc.qc_table_trim(0, 0, t, 1, 0, 0)) == status


@pytest.mark.parametrize("n,ids,new,most,starts,slots,status", [
    (0, 0, 0, 1, 64, 64, 1), (5, 0, 0, 5, 64, 64, 1), (-1, 64, 0, 1, 64, 64, 1), (qc.QC_TABLE_MAX_BATCH + 1, 64, 0, 1, 64, 64, 2), (1, 66, 0, 1, 64, 64, 1),
    (1, 64, 65, 1, 64, 64, 1), (1, 64, 0, -1, 64, 64, 1), (1, 64, 0, 1, 0, 64, 1), (1, 64, 0, 1, 64, 0, 1), (1, 64, 0, 1, 64, 66, 1),
])
def test_a_list_that_is_none_is_refused(n, ids, new, most, starts, slots, status):
    t = qc.qc_table(**OK_TABLE)
    assert status_of(lambda: qc.qc_table_extend(0, 0, t, n, ids, new, most, starts, slots)) == status
    if most == 1 and starts == slots == 64:
        assert status_of(lambda: qc.qc_table_trim(0, 0, t, n, ids, new)) == status


SHAPE = dict(n_kv_heads=2, head_dim=128, page_size=16, n_pages=5)


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=96), 2), (dict(head_dim=0), 2), (dict(page_size=8), 2), (dict(page_size=128), 2), (dict(n_kv_heads=0), 1), (dict(n_pages=0), 1),
    (dict(n_kv_heads=qc.QC_QUANT_MAX_HEADS + 1), 2), (dict(n_pages=1 << 27), 2),
])
def test_a_shape_that_is_none_is_refused(change, status):
    s = qc.qc_quant_shape(**{**SHAPE, **change})
    assert status_of(lambda: qc.qc_quant_pool_bytes(s)) == status
    assert status_of(lambda: qc.qc_quant_append(0, 0, s, 1, 64, 64, 256, 64, 256, 64, 64)) == status
    assert status_of(lambda: qc.qc_quant_read(0, 0, s, 1, 64, 64, 64, 64, 64)) == status


def test_more_tokens_than_indexes_reach_are_refused():
    t, s, n = qc.qc_table(**OK_TABLE), qc.qc_quant_shape(**SHAPE), qc.QC_QUANT_MAX_TOKENS + 1
    assert status_of(lambda: qc.qc_table_extend(0, 0, t, 1, 0, 0, n, 64, 64)) == qc.QC_ERR_UNSUPPORTED
    assert status_of(lambda: qc.qc_quant_append(0, 0, s, n, 64, 64, 256, 64, 256, 64, 64)) == qc.QC_ERR_UNSUPPORTED
    assert status_of(lambda: qc.qc_quant_read(0, 0, s, n, 64, 64, 64, 64, 64)) == qc.QC_ERR_UNSUPPORTED


def test_pool_bytes_and_row_arguments():
    s = qc.qc_quant_shape(**SHAPE)
    assert qc.qc_quant_pool_bytes(s) == 5 * 2 * 16 * 68
    append = lambda n=1, slots=64, k=64, ks=256, v=64, vs=256, kp=64, vp=64: status_of(lambda: qc.qc_quant_append(0, 0, s, n, slots, k, ks, v, vs, kp, vp))
    read = lambda n=1, slots=64, kp=64, vp=64, k=64, v=64: status_of(lambda: qc.qc_quant_read(0, 0, s, n, slots, kp, vp, k, v))
    assert append(n=0, slots=0) == qc.QC_OK and read(n=0, slots=0) == qc.QC_OK
    for bad in (dict(n=-1), dict(slots=0), dict(slots=66), dict(k=0), dict(kp=0), dict(v=0), dict(vp=0), dict(k=0, kp=0, v=0, vp=0), dict(k=72), dict(v=72),
                dict(kp=72), dict(vp=72), dict(ks=-8), dict(vs=-8), dict(ks=4), dict(vs=255)):
        assert append(**bad) == qc.QC_ERR_INVALID_ARG, bad
        if not {"ks", "vs"} & set(bad):
            assert read(**bad) == qc.QC_ERR_INVALID_ARG, bad
    for at in range(4):
        pointers = [64, 64, 64, 64]
        pointers[at] = b"0123456789abcdef"
        with pytest.raises(TypeError):
            qc.qc_quant_read(0, 0, s, 1, 64, *pointers)


def attend_args(stream=None, visual=None, **change):
    t = qc.qc_quant_stream(**{**dict(q_dev=64, q_stride=512, k_pool_dev=64, v_pool_dev=64, pages_dev=64, lens_dev=64, max_pages=4, n_pages=9), **(stream or {})})
    v = qc.qc_quant_stream(**{**dict(q_dev=64, q_stride=512, k_pool_dev=64, v_pool_dev=64, pages_dev=64, lens_dev=64, max_pages=4, n_pages=9), **visual}) if visual is not None else None
    a = qc.qc_quant_attend_args(n_q_heads=4, n_kv_heads=2, head_dim=128, page_size=16, n_seqs=2, max_seqs=3, n_tokens=2, max_queries=1, causal=1,
                                text=t, out_dev=64, workspace_dev=256, workspace_bytes=1 << 40)
    if v is not None:
        a.visual = v
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=80), 2), (dict(page_size=48), 2), (dict(n_q_heads=5), 1), (dict(n_q_heads=0), 1), (dict(n_kv_heads=0), 1), (dict(n_seqs=0), 1), (dict(max_seqs=0), 1),
    (dict(n_seqs=4), 1), (dict(n_tokens=-1), 1), (dict(n_tokens=1), 1), (dict(max_queries=0), 1), (dict(max_queries=qc.QC_QUANT_MAX_QUERIES + 1), 2),
    (dict(n_seqs=qc.QC_QUANT_MAX_SEQS + 1, seq_ids_dev=64), 2), (dict(n_q_heads=2 * qc.QC_QUANT_MAX_HEADS), 2), (dict(text=qc.qc_quant_stream()), 1), (dict(out_dev=0), 1), (dict(out_dev=72), 1),
    (dict(lse_out_dev=66), 1), (dict(status_dev=65), 1), (dict(seq_ids_dev=66), 1), (dict(starts_dev=66), 1), (dict(softmax_scale=-1.0), 1),
    (dict(softmax_scale=math.nan), 1), (dict(softmax_scale=math.inf), 1), (dict(workspace_dev=72), 1),
    (dict(stream=dict(q_dev=0)), 1), (dict(stream=dict(q_dev=72)), 1), (dict(stream=dict(q_stride=-8)), 1), (dict(stream=dict(q_stride=12)), 1), (dict(stream=dict(k_pool_dev=0)), 1),
    (dict(stream=dict(v_pool_dev=24)), 1), (dict(stream=dict(pages_dev=0)), 1), (dict(stream=dict(lens_dev=62)), 1), (dict(stream=dict(max_pages=0)), 1),
    (dict(stream=dict(n_pages=0)), 1), (dict(stream=dict(max_pages=1 << 27)), 2), (dict(stream=dict(n_pages=1 << 27)), 2), (dict(visual=dict(q_dev=0)), 1),
    (dict(visual=dict(max_pages=0)), 1), (dict(visual=dict(n_pages=1 << 28)), 2),
])
def test_attention_refuses_what_it_can_see_on_the_host(change, status):
    assert status_of(lambda: qc.qc_quant_attend(0, 0, attend_args(**change))) == status


def test_attention_refuses_a_workspace_that_is_too_small():
    a = attend_args(stream=dict(max_pages=4000))
    need = qc.qc_quant_workspace_bytes(a)
    assert need > 0
    for size, at in ((need - 1, 256), (need, 0)):
        a.workspace_bytes, a.workspace_dev = size, at
        assert status_of(lambda: qc.qc_quant_attend(0, 0, a)) == qc.QC_ERR_INVALID_ARG


def test_null_pointers_are_refused(lib):
    n = C.c_size_t()
    assert lib.qc_table_reset(0, None, None) == lib.qc_table_trim(0, None, None, 1, None, None) == qc.QC_ERR_INVALID_ARG
    assert lib.qc_quant_pool_bytes(None, C.byref(n)) == lib.qc_quant_pool_bytes(qc.qc_quant_shape(**SHAPE), None) == qc.QC_ERR_INVALID_ARG
    assert lib.qc_quant_attend(0, None, None) == lib.qc_quant_workspace_bytes(None, C.byref(n)) == qc.QC_ERR_INVALID_ARG


def test_without_a_device_a_good_call_is_an_error_status():
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    t, s = qc.qc_table(**OK_TABLE), qc.qc_quant_shape(**SHAPE)
    for call in (lambda: qc.qc_table_reset(0, 0, t), lambda: qc.qc_table_extend(0, 0, t, 1, 0, 0, 1, 64, 64), lambda: qc.qc_table_trim(0, 0, t, 1, 0, 0),
                 lambda: qc.qc_quant_append(0, 0, s, 1, 64, 64, 256, 64, 256, 64, 64), lambda: qc.qc_quant_read(0, 0, s, 1, 64, 64, 64, 64, 64),
                 lambda: qc.qc_quant_attend(0, 0, attend_args())):
        assert status_of(call) == qc.QC_ERR_CUDA


def test_host_tensors_are_refused():
    x, slots = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(1, 16 * 36, dtype=torch.uint8)
    for call in (lambda: quant.append(pool, pool, slots, x, x, 16), lambda: quant.read(pool, pool, slots, 1, 64, 16),
                 lambda: quant.PageTable(slots[None], slots, slots, slots, 16), lambda: quant.attend(quant.Stream(x, pool, pool, slots[None], slots), 1, 16)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError):
        quant.append(None, None, slots, None, None, 16)
    with pytest.raises(ValueError):
        quant.append(pool, None, slots, None, x, 16)
    assert quant.page_bytes(3, 128, 32) == 3 * 32 * 68
