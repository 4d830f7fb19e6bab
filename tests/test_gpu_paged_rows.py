"""Norm and rotation of query and key rows, to tensors and to bf16 pages, against the oracle in 64 bits."""

import math

import numpy as np
import pytest
import torch

from paged_util import DEV, check_rows, gen, rotation, rows
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu


def weight(d, g, kind):
    w = 1 + 0.3 * torch.randn(d, generator=g)
    return None if kind is None else w.to(torch.bfloat16 if kind == "bf16" else torch.float32)


@pytest.mark.parametrize("n,hq,hk,d,rotary,axes,adjacent,norm", [
    (1, 28, 4, 128, 128, 3, False, "bf16"), (1, 1, 1, 64, 64, 1, False, None), (3, 5, 3, 128, 64, 2, True, "f32"), (37, 16, 16, 64, 32, 2, True, "bf16"),
    (150, 32, 32, 128, 128, 3, False, None), (33, 7, 1, 128, 32, 4, False, "f32"), (40, 3, 1, 64, 16, 1, True, None), (5, 12, 2, 128, 16, 2, False, "bf16"),
    (700, 28, 4, 128, 128, 3, False, "bf16"), (1500, 1, 1, 64, 64, 3, True, "f32"), (9, 0, 6, 64, 64, 2, False, "bf16"), (9, 6, 0, 128, 96, 2, False, "bf16"),
    (2, 1024, 1024, 64, 64, 1, False, None), (20, 1024, 37, 128, 128, 2, True, "bf16"), (17, 4, 2, 64, 0, 1, False, "f32"),
])
def test_rows(n, hq, hk, d, rotary, axes, adjacent, norm):
    g = gen(n * hq + hk + d)
    q, k = rows(n, max(1, hq), d, g) if hq else None, rows(n, max(1, hk), d, g) if hk else None
    wq, wk = weight(d, g, norm), weight(d, g, norm)
    positions = torch.randint(-50, 200000, (axes, n), generator=g, dtype=torch.int32)
    rot, freqs, of = rotation(rotary, axes, g, adjacent) if rotary else (None, [], [])
    dev = lambda t: None if t is None else t.to(DEV)
    a, b = paged.rotate(dev(q), dev(k), dev(positions if axes > 1 else positions[0]) if rotary else None, rot, q_norm=dev(wq), k_norm=dev(wk), eps=1e-5)
    for x, got, w in ((q, a, wq), (k, b, wk)):
        if x is None:
            assert got is None
        else:
            check_rows(got, x, positions.tolist(), freqs, of, adjacent, None if w is None else w.double().numpy(), 1e-5)


@pytest.mark.parametrize("n,hq,hk,d", [(400, 150, 150, 128), (3000, 9, 8, 64), (8000, 1, 1, 128)])
def test_rows_of_a_token_in_chunks(n, hq, hk, d):
    """Many tokens of many heads: several warps a token, chunks that begin among the queries and end among the keys."""
    test_rows(n, hq, hk, d, d, 2, False, "bf16")


def test_only_one_of_the_norms():
    g = gen(5)
    q, k, w = rows(6, 2, 128, g), rows(6, 2, 128, g), weight(128, g, "bf16")
    positions = torch.arange(6, dtype=torch.int32)[None]
    rot, freqs, of = rotation(128, 1, g)
    for wq, wk in ((w, None), (None, w)):
        a, b = paged.rotate(q.to(DEV), k.to(DEV), positions.to(DEV), rot, q_norm=None if wq is None else w.to(DEV), k_norm=None if wk is None else w.to(DEV), eps=0.0)
        for x, got, y in ((q, a, wq), (k, b, wk)):
            check_rows(got, x, positions.tolist(), freqs, of, False, None if y is None else y.double().numpy(), 0.0)


@pytest.mark.parametrize("theta", [2.0, 10000.0, 1e7])
def test_far_positions(theta):
    """The rotation of a position is exact however far it is: angles are counted in turns, in 64 bits."""
    g = gen(11)
    at = [0, 1, -1, 12345, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 1000003]
    x = rows(len(at), 2, 64, g)
    freqs = (theta ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    freqs[3], freqs[9], freqs[10] = 123.25, -0.75, 0.0
    rot = paged.Rotation(freqs.to(DEV))
    got, _ = paged.rotate(x.to(DEV), None, torch.tensor(at, dtype=torch.int32, device=DEV), rot)
    # (turns are off by 2^-54 of a frequency's times the position, 2^31 at most, and the oracle's remainder of a product of 24 and 31 bits by 2^-52 of it)
    check_rows(got, x, [at], freqs.tolist(), [0] * 32, False, None, 0.0)


def test_pairs_without_an_axis_or_a_number_are_nan_and_the_others_as_ever():
    g = gen(12)
    x = rows(4, 3, 64, g)
    rot, freqs, of = rotation(64, 2, g)
    positions = torch.randint(0, 100, (2, 4), generator=g, dtype=torch.int32).to(DEV)
    want, _ = paged.rotate(x.to(DEV), None, positions, rot)
    axes, f = rot.axes.clone(), rot.freqs.clone()
    axes[3], axes[7], f[11], f[12] = 2, -1, math.inf, math.nan
    got, _ = paged.rotate(x.to(DEV), None, positions, paged.Rotation(f, axes))
    bad = torch.zeros(64, dtype=torch.bool)
    for pair in (3, 7, 11, 12):
        bad[pair] = bad[pair + 32] = True
    assert got[..., bad].isnan().all() and torch.equal(got[..., ~bad], want[..., ~bad])


def test_infinities_and_nan_stay_in_their_rows():
    g = gen(13)
    x, w = rows(8, 4, 128, g), weight(128, g, "f32")
    y = x.clone()
    y[2, 1, 5], y[3, 2, 77], y[4, 0, 0], y[5, 3] = math.inf, math.nan, -math.inf, 0.0
    rot, freqs, of = rotation(64, 1, g)
    positions = torch.arange(8, dtype=torch.int32, device=DEV)
    for norm in (None, w.to(DEV)):
        a, _ = paged.rotate(x.to(DEV), None, positions, rot, q_norm=norm)
        b, _ = paged.rotate(y.to(DEV), None, positions, rot, q_norm=norm)
        same = torch.ones(8, 4, dtype=torch.bool)
        same[2, 1] = same[3, 2] = same[4, 0] = same[5, 3] = False
        assert torch.equal(a[same], b[same]) and not b[~same][:3].isfinite().all() and (b[5, 3] == 0).all()
        # (without a norm only the pair of such an element is touched)
        if norm is None:
            assert (b[2, 1].isfinite() == torch.tensor([e not in (5, 37) for e in range(128)], device=DEV)).all()


def test_in_place_and_inside_a_fused_projection():
    g = gen(14)
    fused = rows(21, 6 + 2 + 2, 128, g).to(DEV)
    q, k = fused[:, :6], fused[:, 6:8]
    rot, _, _ = rotation(128, 3, g)
    w = weight(128, g, "bf16").to(DEV)
    positions = torch.randint(0, 1000, (3, 21), generator=g, dtype=torch.int32).to(DEV)
    a, b = paged.rotate(q, k, positions, rot, q_norm=w, k_norm=w)
    assert a.is_contiguous() and b.is_contiguous()
    before = fused.clone()
    c, d = paged.rotate(q, k, positions, rot, q_norm=w, k_norm=w, q_out=q, k_out=k)
    assert c.data_ptr() == q.data_ptr() and torch.equal(fused[:, :6], a) and torch.equal(fused[:, 6:8], b) and torch.equal(fused[:, 8:], before[:, 8:])


def test_one_row_for_all_tokens_and_transposed_positions_are_told_apart():
    g = gen(15)
    one = rows(1, 2, 64, g).to(DEV)
    rot, freqs, of = rotation(64, 2, g)
    positions = torch.randint(0, 1000, (9, 2), generator=g, dtype=torch.int32).to(DEV)
    with pytest.raises(ValueError, match="dense"):
        paged.rotate(one.expand(9, 2, 64), None, positions.T, rot)
    wide = torch.zeros(2, 20, dtype=torch.int32, device=DEV)
    wide[:, :9] = positions.T
    got, _ = paged.rotate(one.expand(9, 2, 64), None, wide[:, :9], rot)
    check_rows(got, one.cpu().expand(9, 2, 64), positions.T.tolist(), freqs, of, False, None, 0.0)


# ---- to the pages -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,hq,hk,d,page,norm,what", [
    (1, 28, 4, 128, 16, "bf16", "qkv"), (32, 28, 4, 128, 16, None, "qkv"), (70, 3, 5, 64, 32, "f32", "qkv"), (131, 4, 4, 128, 64, "bf16", "kv"),
    (50, 8, 2, 64, 16, None, "k"), (50, 8, 2, 128, 32, None, "v"), (50, 8, 2, 64, 64, "bf16", "qv"), (900, 8, 2, 128, 16, "bf16", "qkv"),
])
def test_rows_go_to_their_slots_and_nothing_else_changes(n, hq, hk, d, page, norm, what):
    g = gen(n + d)
    q, k, v = rows(n, hq, d, g), rows(n, hk, d, g), rows(n, hk, d, g)
    w = weight(d, g, norm)
    w = None if w is None else w.to(DEV)
    rot, _, _ = rotation(d, 3, g, adjacent=page == 32)
    positions = torch.randint(0, 100000, (3, n), generator=g, dtype=torch.int32).to(DEV)
    n_pages = n // page + 4
    slots = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
    slots[torch.rand(n, generator=g) < 0.2] = -1
    if n > 40:
        slots[5], slots[17], slots[18] = n_pages * page, 2 ** 31 - 1, -2 ** 31      # not in the pool
    pools = [torch.randn(n_pages, hk, page, d, generator=g).bfloat16().to(DEV) for _ in "kv"]
    before = [p.clone() for p in pools]
    there = (slots >= 0) & (slots < n_pages * page)
    with_k, with_v = "k" in what, "v" in what
    got = paged.append(pools[0] if with_k else None, pools[1] if with_v else None, slots.to(DEV), k.to(DEV) if with_k else None, v.to(DEV) if with_v else None,
                       q=q.to(DEV) if "q" in what else None, positions=positions, rotation=rot, q_norm=w, k_norm=w)
    want_q, want_k = paged.rotate(q.to(DEV), k.to(DEV), positions, rot, q_norm=w, k_norm=w)
    assert torch.equal(got, want_q) if "q" in what else got is None
    at = slots[there].long().to(DEV)
    if with_k:
        before[0][at // page, :, at % page] = want_k[there.to(DEV)]
    if with_v:
        before[1][at // page, :, at % page] = v.to(DEV)[there.to(DEV)]
    assert torch.equal(pools[0], before[0]) and torch.equal(pools[1], before[1])


def test_a_pool_past_32_bits_of_elements():
    """Element 2^31 and beyond of a pool: 33 000 pages of 32 heads of 16 tokens."""
    n_pages, page = 33000, 16
    pool = torch.zeros(n_pages, 32, page, 128, dtype=torch.bfloat16, device=DEV)
    assert pool.numel() > 2 ** 31
    v = rows(3, 32, 128, gen(21)).to(DEV)
    slots = torch.tensor([n_pages * page - 1, (n_pages - 300) * page, 5], dtype=torch.int32, device=DEV)
    paged.append(None, pool, slots, None, v)
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(pool[s // page, :, s % page], v[i])
    assert int((pool != 0).any(-1).sum()) == 3 * 32


def test_no_tokens():
    x, pool = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV), torch.ones(1, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    rot, _, _ = rotation(64, 1, gen(1))
    a, b = paged.rotate(x, x, none, rot)
    assert a.shape == b.shape == x.shape
    assert paged.append(pool, pool.clone(), none, x, x, q=x, positions=none, rotation=rot).shape == x.shape and (pool == 1).all()


def test_a_captured_step_takes_new_positions_and_slots_in_its_replays():
    g = gen(22)
    n, hq, hk, d, page = 5, 8, 2, 128, 16
    rot, _, _ = rotation(d, 2, g)
    fused = torch.empty(n, hq + 2 * hk, d, dtype=torch.bfloat16, device=DEV)
    positions, slots = torch.zeros(2, n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    pools = [torch.zeros(4, hk, page, d, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    step = lambda q_out=None: paged.append(*pools, slots, fused[:, hq:hq + hk], fused[:, hq + hk:], q=fused[:, :hq], positions=positions, rotation=rot, q_out=q_out)
    fused.copy_(rows(n, hq + 2 * hk, d, g))
    slots.copy_(torch.arange(n, dtype=torch.int32))
    step()
    q_out = torch.empty(n, hq, d, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(q_out)
    for i in range(3):
        fused.copy_(rows(n, hq + 2 * hk, d, g))
        positions.copy_(torch.randint(0, 1000, (2, n), generator=g, dtype=torch.int32))
        slots.copy_(torch.randperm(64, generator=g)[:n].to(torch.int32))
        graph.replay()
        got, held = q_out.clone(), [p.clone() for p in pools]
        for p in pools:
            p[slots.long() // page, :, slots.long() % page] = 0
        assert torch.equal(step(), got) and all(torch.equal(a, b) for a, b in zip(pools, held))


def test_another_stream_than_the_tensors_own():
    g = gen(23)
    x = rows(2000, 16, 128, g)
    rot, freqs, of = rotation(128, 1, g)
    positions = torch.arange(2000, dtype=torch.int32, device=DEV)
    want, _ = paged.rotate(x.to(DEV), None, positions, rot)
    y = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.copy_(x.to(DEV))
        got, _ = paged.rotate(y, None, positions, rot)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("change", [
    dict(q=lambda q: q.float()), dict(q=lambda q: q[:, :, ::2]), dict(q=lambda q: q[:, ::2]), dict(q=lambda q: q[0]), dict(q=lambda q: q.cpu()), dict(k=lambda k: k[:3]), dict(k=lambda k: k.half()),
    dict(positions=lambda p: p.long()), dict(positions=lambda p: p[:, :3]), dict(positions=lambda p: p.cpu()), dict(positions=lambda p: None), dict(positions=lambda p: p[None]),
    dict(rotation=lambda r: None), dict(rotation=lambda r: r._replace(freqs=r.freqs.double())), dict(rotation=lambda r: r._replace(axes=r.axes.long())),
    dict(rotation=lambda r: r._replace(axes=r.axes[:5])), dict(rotation=lambda r: r._replace(freqs=r.freqs[:12], axes=r.axes[:12])),
    dict(rotation=lambda r: r._replace(freqs=r.freqs.repeat(2), axes=r.axes.repeat(2))), dict(rotation=lambda r: r._replace(freqs=r.freqs[:0], axes=r.axes[:0])), dict(rotation=lambda r: r.freqs),
    dict(q_norm=lambda w: w.half()), dict(q_norm=lambda w: w[:5]), dict(k_norm=lambda w: w.float()), dict(eps=lambda e: -1.0), dict(eps=lambda e: math.nan), dict(q_out=lambda o: torch.zeros(4, 4, 64, device=DEV)),
    dict(q_out=lambda o: torch.zeros(4, 3, 64, dtype=torch.bfloat16, device=DEV)), dict(k_out=lambda o: torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=DEV).expand(4, 2, 64)),
])
def test_what_does_not_fit_is_refused(change):
    g = gen(24)
    rot, _, _ = rotation(64, 2, g)
    args = dict(q=rows(4, 4, 64, g).to(DEV), k=rows(4, 2, 64, g).to(DEV), positions=torch.zeros(2, 4, dtype=torch.int32, device=DEV), rotation=rot,
                q_norm=torch.ones(64, dtype=torch.bfloat16, device=DEV), k_norm=torch.ones(64, dtype=torch.bfloat16, device=DEV), eps=1e-6, q_out=None, k_out=None)
    paged.rotate(**args)
    for name, make in change.items():
        args[name] = make(args[name])
    with pytest.raises((ValueError, qc.QcError)):
        paged.rotate(**args)


@pytest.mark.parametrize("change", [
    dict(k_pool=lambda p: p.float()), dict(k_pool=lambda p: p[:, :1]), dict(k_pool=lambda p: p.transpose(1, 2)), dict(k_pool=lambda p: p[..., :32]), dict(v_pool=lambda p: p[:2]), dict(k_pool=lambda p: None),
    dict(v=lambda v: v[:3]), dict(v=lambda v: v[:, :1]), dict(slots=lambda s: s.long()), dict(slots=lambda s: s[:3]), dict(slots=lambda s: s.cpu()), dict(q=lambda q: q[:2]), dict(q=lambda q: q[..., :32]),
    dict(k_pool=lambda p: torch.zeros(3, 2, 24, 64, dtype=torch.bfloat16, device=DEV), v_pool=lambda p: torch.zeros(3, 2, 24, 64, dtype=torch.bfloat16, device=DEV)),
])
def test_an_append_that_does_not_fit_is_refused(change):
    g = gen(25)
    make_pool = lambda: torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    args = dict(k_pool=make_pool(), v_pool=make_pool(), slots=torch.arange(4, dtype=torch.int32, device=DEV), k=rows(4, 2, 64, g).to(DEV), v=rows(4, 2, 64, g).to(DEV), q=rows(4, 6, 64, g).to(DEV))
    paged.append(**args)
    for name, make in change.items():
        args[name] = make(args[name])
    with pytest.raises((ValueError, qc.QcError)):
        paged.append(**args)
