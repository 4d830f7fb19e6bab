"""Attention over bf16 pages key by key, at lengths that are cut into many pieces: every key counts once, in its own row, for the queries that see it."""

import random

import numpy as np
import pytest
import torch

from paged_marks import SCALE, channel_of, check_counts, counts, marks
from paged_util import DEV, gen
from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import paged

pytestmark = pytest.mark.gpu


def stream_of(rows, n_rows, ids, hkv, d, page, g):
    """A table and pools that hold rows of marks; NaN where no token is."""
    lens = [m.n for m in rows]
    n_pages = sum(-(-n // page) for n in lens) + 2
    table = paged.PageTable.empty(n_rows, max([-(-n // page) for n in lens] + [0]) + 1, page, n_pages)
    table.free.copy_(torch.randperm(n_pages, generator=g).to(torch.int32))
    pools = [torch.full((n_pages, hkv, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    if sum(lens):
        _, slots = paged.table_extend(table, torch.tensor(lens, dtype=torch.int32, device=DEV), seq_ids=ids, max_slots=sum(lens))
        k = torch.zeros(sum(lens), hkv, d, dtype=torch.bfloat16, device=DEV)
        v = torch.zeros_like(k)
        k[:, :, 0] = torch.tensor(np.concatenate([m.doublings for m in rows]), device=DEV)[:, None].bfloat16()
        of = [np.stack([channel_of(m, h, np.arange(m.n)) for h in range(hkv)], 1) for m in rows]
        value = torch.tensor(np.concatenate([np.full(m.n, m.value) for m in rows]), device=DEV).bfloat16()
        v.scatter_(2, torch.tensor(np.concatenate(of), device=DEV)[..., None], value[:, None, None].expand(-1, hkv, 1))
        paged.append(*pools, slots, k, v)
    table.check()
    return table, pools


def run(seed, own, queries, groups, hkv, group, d, page, causal=True, only=None):
    """own: marks of each sequence; queries: how many each has; groups: [(first, last, marks of the prefix)]."""
    g, n = gen(seed), len(own)
    ids = torch.randperm(n + 1, generator=g)[:n].to(torch.int32).to(DEV)
    begin = np.concatenate([[0], np.cumsum(queries)])
    q = torch.zeros(int(begin[-1]), hkv * group, d, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1
    table, pools = stream_of(own, n + 1, ids, hkv, d, page, g)
    kw = {}
    if groups:
        shared_ids = torch.randperm(len(groups) + 1, generator=g)[:len(groups)].to(torch.int32).to(DEV)
        images, image_pools = stream_of([m for _, _, m in groups], len(groups) + 1, shared_ids, hkv, d, page, g)
        kw = dict(shared=paged.Stream(q, *image_pools, images.pages, images.lens), shared_ids=shared_ids,
                  groups=torch.tensor([groups[0][0]] + [b for _, b, _ in groups], dtype=torch.int32, device=DEV))
    out, lse = paged.attend(paged.Stream(q, *pools, table.pages, table.lens), seq_ids=ids, starts=torch.tensor(begin, dtype=torch.int32, device=DEV),
                            max_queries=max(queries), causal=causal, scale=SCALE, status=table.state[1:2], **kw)
    assert int(table.state[1]) == qc.QC_OK
    out, lse = out.double().cpu().numpy(), lse.cpu().numpy()
    for i in range(n) if only is None else only:
        prefix = [(m, m.n) for a, b, m in groups if a <= i < b]
        for j in range(queries[i]):
            parts = prefix + [(own[i], max(0, own[i].n - (queries[i] - 1 - j)) if causal else own[i].n)]
            keys, token = sum(seen for _, seen in parts), begin[i] + j
            for h in range(hkv):
                if keys:
                    total, by = counts(parts, h, d)
                for head in range(h * group, (h + 1) * group):
                    if keys:
                        check_counts(out[token, head], float(lse[token, head]), total, by, keys, (i, j, head))
                    else:
                        assert (out[token, head] == 0).all() and lse[token, head] == -np.inf


@pytest.mark.parametrize("lens,queries,groups,hkv,group,d,page", [
    ([9000, 20011, 1], [1, 3, 2], [(0, 2, 30017)], 1, 4, 128, 64),
    ([9000, 20011, 1], [1, 3, 2], [(0, 2, 30017)], 2, 4, 64, 16),
    ([0] * 19 + [5], [1] * 20, [(0, 20, 40000)], 1, 1, 128, 64),
    ([0] * 19 + [70], [1] * 20, [(0, 20, 19000)], 1, 1, 64, 32),
    ([9000] * 20, [1] * 20, [(0, 20, 1)], 1, 1, 128, 16),
    ([20000] + [0] * 19, [1] * 20, [(0, 20, 65)], 1, 1, 128, 64),
    ([8541] * 8, [1] * 8, [], 4, 1, 128, 16),
    ([50, 200, 3] * 20, [1] * 60, [(2, 59, 32768)], 2, 7, 128, 64),
    ([50, 200, 3] * 20, [1] * 60, [(2, 59, 16385)], 2, 7, 64, 16),
    ([5000, 700, 6001], [16, 17, 15], [(0, 3, 7003)], 2, 1, 128, 16),          # rows of a sequence on both sides of what a warp takes
    ([5000, 700, 6001], [3, 4, 5], [(0, 1, 7003), (1, 3, 901)], 1, 5, 64, 32),
    ([3000, 128, 100, 5003], [128, 128, 128, 77], [(1, 4, 2111)], 1, 2, 128, 32),
])
def test_every_key_counts_once(lens, queries, groups, hkv, group, d, page):
    run(len(lens), [marks(n, 7 * i, 0, d, 3.0) for i, n in enumerate(lens)], queries, [(a, b, marks(p, 3 * a, 0, d)) for a, b, p in groups], hkv, group, d, page)


@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 128, 129, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_every_length_along_a_stretch(rows, d):
    """A prefix that one, two, ... of many workers have, with its borders at every place of a tile."""
    for n in [*range(2049, 2049 + 17 * 9, 17), 6000, 11111]:
        run(n, [marks(n % 90, 3, 0, d, 3.0)] * rows, [1] * rows, [(0, rows, marks(n, 0, 0, d))], 1, 1, d, 16, only=range(0, rows, 29))


@pytest.mark.parametrize("seed", range(24))
def test_batches_of_many_kinds_key_by_key(seed):
    rng = random.Random(seed)
    d, n = rng.choice([64, 128]), rng.choice([1, 3, 9, 40])
    high, pre = rng.choice([40, 700, 9000]), rng.choice([300, 5000, 25000])
    queries = [rng.randint(1, rng.choice([1, 4, 40])) for _ in range(n)]
    cuts = sorted(rng.randint(0, n) for _ in range(rng.choice([0, 2, 4])))
    hkv, group = rng.choice([(1, 1), (2, 7), (4, 2), (1, 16), (3, 5)])
    run(seed, [marks(rng.randint(0, high), 11 * i, 0, d, 3.0) for i in range(n)], queries,
        [(a, b, marks(rng.randint(0, pre), 3 * a, 0, d)) for a, b in zip(cuts, cuts[1:])], hkv, group, d, rng.choice([16, 32, 64]), causal=rng.random() < 0.7,
        only=rng.sample(range(n), min(n, 12)))


@pytest.mark.parametrize("seed", range(16))
def test_weights_far_apart_key_by_key(seed):
    """Pieces of different references: a tile's weights are 2^-12 to 2^12, and each tile has a channel to itself."""
    rng = random.Random(seed)
    d, n = rng.choice([64, 128]), rng.choice([1, 4, 20])
    half, most = d // 2, rng.choice([3, 12, 24])
    make = lambda n, first, value: marks(n, 0, first, half, value, np.array([rng.randint(0, most) - most // 2 for _ in range(-(-n // 16))] or 0))
    queries = [rng.randint(1, rng.choice([1, 6, 30])) for _ in range(n)]
    run(seed, [make(rng.randint(0, half * 16), half, 3.0) for _ in range(n)], queries, [(0, n, make(rng.randint(1, half * 16), 0, 1.0))], *rng.choice([(1, 1), (2, 4), (1, 9)]), d,
        rng.choice([16, 32, 64]), only=rng.sample(range(n), min(n, 8)))
