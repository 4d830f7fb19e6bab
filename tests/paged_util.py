"""Seeded rows, positions and rotations for the tests of rows and bf16 pages, with the oracle's view and how far an output may be off."""

import math

import numpy as np
import torch

from oracle import positions as O
from paper_2602_01901_b200 import paged, quant

DEV = "cuda"


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows(n, heads, head_dim, g):
    """bf16 rows on the CPU: channels and tokens of different size."""
    channel = torch.exp(0.5 * torch.randn(heads, head_dim, generator=g))
    token = torch.exp(0.4 * torch.randn(n, 1, 1, generator=g))
    return (torch.randn(n, heads, head_dim, generator=g) * channel * token).bfloat16()


def rotation(rotary, n_axes, g, adjacent=False, theta=10000.0):
    """(Rotation on the device, frequencies, axes) of `rotary` elements; axes in no order."""
    pairs = rotary // 2
    freqs = (theta ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    axes = torch.randint(0, n_axes, (pairs,), generator=g, dtype=torch.int32)
    return paged.Rotation(freqs.to(DEV), axes.to(DEV) if n_axes > 1 else None, adjacent), freqs.tolist(), axes.tolist() if n_axes > 1 else [0] * pairs


def check_rows(got, x, positions, freqs, axes, adjacent, weight, eps):
    """Rows against the oracle.  x [n, heads, d] bf16 on the CPU, positions [axes, n] integers, freqs empty: no rotation.

    With a norm an element is x * scale * w: the sum of d squares is off by (d + 1) 2^-24 of itself at most, the mean and eps add
    2^-23, the reciprocal root halves that and adds 2^-22, and two products 2^-24 each.  An angle is cut off at 2^-32 turns and
    rounded to 2^-24 half turns at most; its sine and cosine are off by 2^-23 more: 2^-21 of the pair's elements together.  Two products and a
    sum round three times, 2^-24 each of |a| + |b|.  Then half a step of bf16, 2^-8."""
    x, got = x.double().numpy(), got.double().cpu().numpy()
    d = x.shape[-1]
    a = O.normed(x, weight, eps)
    want = O.turned(a, positions, freqs, axes, adjacent) if len(freqs) else a
    size = np.abs(a)
    for e in range(2 * len(freqs)):
        size[..., e] = np.abs(a[..., e]) + np.abs(a[..., O.pair_of(e, len(freqs), adjacent)[2]])
    rel = (2.0 ** -21 + 3 * 2.0 ** -24 if len(freqs) else 0.0) + ((d + 3) * 2.0 ** -25 + 2.0 ** -22 + 2.0 ** -23 if weight is not None else 0.0)
    tol = 2.0 ** -8 * np.abs(want) + 2 * rel * size + 2.0 ** -133
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all() and (np.where(fine, 0, got) == np.where(fine, 0, want))[~np.isnan(want)].all()
    far = np.where(fine, np.abs(got - want) / tol, 0)
    assert far.max(initial=0.0) <= 1, (np.unravel_index(far.argmax(), far.shape), far.max())


# ---- batches for attention ---------------------------------------------------------------------------------------

def stream_of(lens, ids, n_rows, hkv, d, page, g, spread=1.0, extra_pages=2):
    """A table and pools with rows of the given lengths in table rows `ids`, NaN where no token is: (table, pools, keys, values), the last
    two lists of [len, heads, d] on the device."""
    lens = list(lens)
    n_pages = sum(-(-n // page) for n in lens) + extra_pages
    table = paged.PageTable.empty(n_rows, max([-(-n // page) for n in lens] + [0]) + 2, page, n_pages)
    # pages in no order
    table.free.copy_(torch.randperm(n_pages, generator=g).to(torch.int32))
    pools = [torch.full((n_pages, hkv, page, d), math.nan, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    ids = torch.tensor(list(ids), dtype=torch.int32, device=DEV)
    keys, values = [[(spread * torch.randn(n, hkv, d, generator=g)).bfloat16().to(DEV) for n in lens] for _ in "kv"]
    if sum(lens):
        _, slots = paged.table_extend(table, torch.tensor(lens, dtype=torch.int32, device=DEV), seq_ids=ids, max_slots=sum(lens))
        paged.append(*pools, slots, torch.cat(keys), torch.cat(values))
    table.check()
    return table, pools, keys, values


class Batch:
    """Sequences of own lengths `lens` and `queries` query tokens each; groups [(first, last, prefix length)]."""

    def __init__(self, seed, lens, queries, groups, hkv, group, d, page, lazy=False, causal=True, scale=0.0, spread=1.0):
        g = gen(seed)
        n, self.d, self.hkv, self.group, self.causal = len(lens), d, hkv, group, causal
        self.scale = scale or 1 / math.sqrt(d)
        self.given_scale, self.lens, self.queries, self.groups, self.page = scale, list(lens), list(queries), list(groups), page
        ids = torch.randperm(n + 2, generator=g)[:n]
        self.ids = ids.to(torch.int32).to(DEV)
        self.table, self.pools, self.keys, self.values = stream_of(lens, ids.tolist(), n + 2, hkv, d, page, g, spread)
        self.begin = [0]
        for q in queries:
            self.begin.append(self.begin[-1] + q)
        tokens = self.begin[-1]
        make_q = lambda: (spread * torch.randn(tokens, hkv * group, d, generator=g)).bfloat16().to(DEV)
        self.q = make_q()
        self.q_shared = make_q() if lazy else self.q
        self.starts = torch.tensor(self.begin, dtype=torch.int32, device=DEV)
        self.shared = None
        if groups:
            shared_ids = torch.randperm(len(groups) + 1, generator=g)[:len(groups)]
            self.shared_ids = shared_ids.to(torch.int32).to(DEV)
            self.group_starts = torch.tensor([groups[0][0]] + [b for _, b, _ in groups], dtype=torch.int32, device=DEV)
            self.shared = stream_of([p for _, _, p in groups], shared_ids.tolist(), len(groups) + 1, hkv, d, page, g, spread)

    def stream(self):
        return paged.Stream(self.q, *self.pools, self.table.pages, self.table.lens)

    def shared_stream(self):
        table, pools, _, _ = self.shared
        return paged.Stream(self.q_shared, *pools, table.pages, table.lens)

    def call(self, **change):
        args = dict(seq_ids=self.ids, starts=self.starts, max_queries=max(1, max(self.queries)), causal=self.causal, scale=self.given_scale, status=self.table.state[1:2])
        if self.shared is not None:
            args.update(shared=self.shared_stream(), groups=self.group_starts, shared_ids=self.shared_ids)
        args.update(change)
        return paged.attend(args.pop("own", None) or self.stream(), **args)

    def parts(self, i):
        """(queries, keys, values, keys seen by each query) of the streams that sequence i sees."""
        a, b = self.begin[i], self.begin[i + 1]
        n = self.lens[i]
        place = torch.arange(b - a, device=DEV)
        own = (self.q[a:b], self.keys[i], self.values[i], (n - (b - a - 1) + place).clamp(min=0) if self.causal else torch.full_like(place, n))
        for j, (first, last, p) in enumerate(self.groups):
            if first <= i < last:
                return [(self.q_shared[a:b], self.shared[2][j], self.shared[3][j], torch.full_like(place, p)), own]
        return [own]

    def check(self, out, lse, only=None):
        for i in range(len(self.lens)) if only is None else only:
            a, b = self.begin[i], self.begin[i + 1]
            if a < b:
                check_rows_of(out[a:b], lse[a:b], self.parts(i), self.group, self.scale, f"sequence {i}")


def attention(parts, group, scale):
    """In 64 bits: (out [queries, heads, d], lse [queries, heads], weights' mass sum w |v|, largest error of a score over 2^-23, n)."""
    logits, sizes, values = [], [], []
    for q, k, v, seen in parts:
        n, heads, d = q.shape
        x = q.double().reshape(n, heads // group, group, d)
        k, v = k.double(), v.double()
        there = torch.arange(k.shape[0], device=DEV) < seen[:, None]
        dot = torch.einsum("qhgd,lhd->qhgl", x, k) * scale
        logits.append(torch.where(there[:, None, None], dot, -math.inf))
        sizes.append(torch.where(there[:, None, None], torch.einsum("qhgd,lhd->qhgl", x.abs(), k.abs()) * scale, 0.0))
        values.append(v)
    logit, size, v = torch.cat(logits, -1), torch.cat(sizes, -1), torch.cat(values)
    n, hkv, group, keys = logit.shape
    if keys == 0:
        zero = torch.zeros(n, hkv * group, v.shape[-1], dtype=torch.float64, device=DEV)
        return zero, torch.full(zero.shape[:2], -math.inf, dtype=torch.float64, device=DEV), zero, zero[..., 0], 0
    lse = torch.logsumexp(logit, -1)
    w = torch.where(lse[..., None].isfinite(), torch.exp(logit - lse[..., None]), 0.0)
    flat = lambda t: t.reshape(n, hkv * group, *t.shape[3:])
    out, mass = torch.einsum("qhgl,lhd->qhgd", w, v), torch.einsum("qhgl,lhd->qhgd", w, v.abs())
    return flat(out), flat(lse), flat(mass), flat(size.amax(-1)), keys


def check_rows_of(out, lse, parts, group, scale, where):
    """Output rows of a sequence against softmax attention in 64 bits.

    A score is a sum of d exact products in fp32: every addition is off by 2^-23 (an adder that cuts off) of the sum of the
    magnitudes at most, as are the scaling and the difference to the reference: e = (d + 4) 2^-23 sum |q k| scale.  The exponential adds 2^-22
    of itself and a rounding of its argument, 2^-24 of at most 2^7, whose weight is 2^-100 there: 2^-22 where it counts.  Weights are
    rounded to bf16 for the value product (2^-8 of themselves), their sum is not; sums over n keys in fp32 are off by 2^-23 per
    step.  The output is rounded to bf16, 2^-8 of itself."""
    want, want_lse, mass, size, n = attention(parts, group, scale)
    d = want.shape[-1]
    e = size * (d + 4) * 2.0 ** -23
    rel = 2 * e + 2.0 ** -20 + (n + 64) * 2.0 ** -23
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -8 * (1 + 2.0 ** -7) + 2 * rel)[..., None] * mass + 1e-37
    far = (out.double() - want).abs() - tol
    assert not (far > 0).any() and not out.isnan().any(), (where, (far > 0).nonzero()[:5].tolist(), far.max().item())
    some = want_lse.isfinite()
    assert (lse[~some] == -math.inf).all() and (out[~some] == 0).all(), where
    off = (lse.double() - want_lse).abs() - (e + 2.0 ** -20 + (n + 64) * 2.0 ** -23 + 2.0 ** -23 * want_lse.abs())
    assert not (off[some] > 0).any(), (where, off[some].max().item())
