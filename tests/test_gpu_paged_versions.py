"""Tensors that the calls on positions and bf16 pages write to count as changed: a graph that has kept one says so instead of using it."""

import pytest
import torch

from paged_util import DEV, Batch, gen, rotation, rows
from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu


def changed(tensors, call):
    before = [t._version for t in tensors]
    call()
    return [t._version > v for t, v in zip(tensors, before)]


def test_what_is_written_counts_as_changed_and_nothing_else():
    g = gen(1)
    fused, slots = rows(4, 6, 64, g).to(DEV), torch.arange(4, dtype=torch.int32, device=DEV)
    q, k, v = fused[:, :2], fused[:, 2:4], fused[:, 4:]
    rot, _, _ = rotation(64, 1, g)
    q_out, pools = torch.empty(4, 2, 64, dtype=torch.bfloat16, device=DEV), [torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    assert changed([fused, q_out, slots], lambda: paged.rotate(q, k, slots, rot)) == [False] * 3
    assert changed([fused, q_out, slots], lambda: paged.rotate(q, k, slots, rot, q_out=q_out)) == [False, True, False]
    assert changed([fused, q_out, slots], lambda: paged.rotate(q, k, slots, rot, q_out=q, k_out=k)) == [True, False, False]
    assert changed([fused, *pools], lambda: paged.append(*pools, slots, k, v, q=q)) == [False, True, True]
    assert changed([fused, *pools, q_out], lambda: paged.append(None, pools[1], slots, None, v, q=q, q_out=q_out)) == [False, False, True, True]
    b = Batch(1, [5, 60], [1, 1], [(0, 2, 9)], 2, 2, 64, 16)
    out = torch.empty_like(b.q)
    assert changed([b.q, *b.pools, out], lambda: b.call(out=out)) == [False, False, False, True]


def test_a_graph_that_kept_what_was_turned_in_place_says_so():
    g = gen(2)
    x = rows(4, 2, 64, g).float().to(DEV).requires_grad_()
    q = x.bfloat16()
    total = (q * q).sum()
    rot, _, _ = rotation(64, 1, g)
    with torch.no_grad():
        paged.rotate(q, None, torch.arange(4, dtype=torch.int32, device=DEV), rot, q_out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        total.backward()


def test_tensors_of_inference_mode_count_nothing():
    g = gen(3)
    with torch.inference_mode():
        q, slots = rows(4, 2, 64, g).to(DEV), torch.arange(4, dtype=torch.int32, device=DEV)
        pool = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
        rot, _, _ = rotation(64, 1, g)
        want = paged.rotate(q, None, slots, rot)[0]
        paged.append(pool, None, slots, q, None, positions=slots, rotation=rot)
        assert paged.rotate(q, None, slots, rot, q_out=q)[0] is not None and torch.equal(q, want) and torch.equal(pool[0, :, :4].transpose(0, 1), want)
