"""Seeded caches in 4 bits for the tests, with the oracle's view of what they hold and how far an output may be off."""

import math

import numpy as np
import torch

from oracle import quant_cache as O
from paper_2602_01901_b200 import quant

DEV = "cuda"


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows(n, heads, head_dim, g, spread=1.0):
    """bf16 rows on the CPU: channels and tokens of different size."""
    channel = torch.exp(0.5 * spread * torch.randn(heads, head_dim, generator=g))
    token = torch.exp(0.4 * spread * torch.randn(n, 1, 1, generator=g))
    return (torch.randn(n, heads, head_dim, generator=g) * channel * token).bfloat16()


def held(x):
    """What the cache holds of bf16 rows [n, heads, head_dim]: fp64 lo, step, codes, values, by the oracle's rule row by row."""
    a = x.double().numpy().reshape(-1, x.shape[-1])
    lo, step, codes = np.empty(len(a)), np.empty(len(a)), np.empty(a.shape)
    for i, row in enumerate(a):
        lo[i], r, codes[i] = O.quantise(row)
        step[i] = 1.0 / r if r else 0.0
    lead = x.shape[:-1]
    lo, step, codes = lo.reshape(lead), step.reshape(lead), codes.reshape(x.shape)
    return {"lo": lo, "step": step, "codes": codes, "values": lo[..., None] + step[..., None] * codes}


def fill(table, ids, lens, page, pools, k, v, device=DEV):
    """Stores rows k, v (lists of bf16 [len, heads, head_dim], one per sequence) in one call."""
    n_new = torch.tensor(lens, dtype=torch.int32, device=device)
    starts, slots = quant.table_extend(table, n_new, seq_ids=ids, max_slots=sum(lens))
    if sum(lens):
        quant.append(pools[0], pools[1], slots, torch.cat(k).to(device), torch.cat(v).to(device), page)
    return starts, slots


def bound(queries, keys, values, scale, out, weights):
    """How far an output row may be from the one in 64 bits, element by element, and its lse; `weights`: the softmax's.

    A score is s * sum q c + lo * sum q.  A query element is exact in fp16 with the largest of the rows computed together in
    2^14 .. 2^15 (half of them divided by 16 before), or off by half of the least step, 2^-25 times 16: by 2^-35 of that largest
    one at most.  The products are exact and summed in fp32: every one of the D + 8 steps is off by 2^-23 of the sum's largest
    magnitude at most (an adder that cuts off), as are the four roundings around it; |score| is bounded with absolute values.
    The exponential adds 2^-22 of itself and the rounding of its argument.  The weights p s are rounded to fp16 (2^-11) before
    the product with c - 8; the sums over L keys, in fp32, are off by 2^-23 per step of what they add up; s in lo + 8 s is off by
    2^-23 of itself, 2^-20 p s; the output is rounded to bf16 (2^-8).

    The adder lines up 16 addends and the sum so far by the operands' exponents, a subnormal code's being that of 2^-14: each
    addend is cut off at 2^-15 of the largest query element (scores) or weight p s (values) among the 16, times one code.  An
    addend whose factor is not below 2^-7 of the largest query element (8 bits) or 2^-4 of the largest weight (11 bits) has nothing
    there; another loses no more than it is, 15 times the factor.  The codes' addends and those that take off the 8 are cut
    off in opposite directions.  The sum so far is cut off D / 16 times for a score and eight times for a tile of 64 values.
    """
    n = sum(len(k["step"]) for k in keys)
    e = 0.0
    for q, k in zip(queries, keys):
        if len(k["step"]):
            part = k["codes"] @ np.abs(q) * k["step"] + np.abs(k["lo"]) * np.abs(q).sum()
            top = np.abs(q).max()
            small = np.where(np.abs(q) < 2.0 ** -7 * top, np.minimum(2.0 ** -15 * top, 15 * np.abs(q)), 0.0).sum()
            cut = k["step"] * (small + (q.size / 16 * 2.0 ** -15 * top if small else 0.0))
            e = max(e, scale * float((part * (q.size + 12) * 2.0 ** -23 + cut).max()))
    size = np.concatenate([np.abs(v["lo"] + 8 * v["step"])[:, None] + v["step"][:, None] * np.abs(v["codes"] - 8) for v in values]) if n else np.zeros((1, out.size))
    mass = weights @ size if n else np.zeros(out.size)
    ps = weights * np.concatenate([v["step"] for v in values]) if n else np.zeros(1)
    cut = np.minimum(2.0 ** -15 * ps.max(), 15 * ps).sum() + 2.0 ** -12 * min((n / 64 + 2) * ps.max(), ps.sum())
    rel = 2 * e + 2.0 ** -21 + (n + 64) * 2.0 ** -23
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + 2 * rel) * mass + cut + 2.0 ** -20 * ps.sum() + 1e-37, e + 2.0 ** -20 + (n + 64) * 2.0 ** -23


def check_attend(out, lse, starts, ids, lens, q, k_held, v_held, group, scale, causal=True, visual=None):
    """Every output row against the oracle.  q bf16 [tokens, heads, d] on the CPU; k_held, v_held: per sequence what
    ``held`` gives; visual: (q, k_held, v_held)."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    qs = q.double().numpy()
    heads = qs.shape[1]
    cut = lambda h, n, kvh: {name: a[:n, kvh] for name, a in h.items()}
    for i in range(len(lens)):
        a, b = starts[i], starts[i + 1]
        for t in range(a, b):
            seen = max(0, lens[i] - (b - 1 - t)) if causal else lens[i]
            for h in range(heads):
                kvh = h // group
                keys, values, queries = [cut(k_held[i], seen, kvh)], [cut(v_held[i], seen, kvh)], [qs[t, h]]
                if visual is not None:
                    n = len(visual[1][i]["lo"])
                    keys.append(cut(visual[1][i], n, kvh)), values.append(cut(visual[2][i], n, kvh)), queries.append(visual[0].double().numpy()[t, h])
                streams = [(x, k["values"], v["values"]) for x, k, v in zip(queries, keys, values)]
                want, want_lse = O.attention(qs[t, h], streams, scale)
                where = f"sequence {i} query {t - a} head {h}"
                if not np.isfinite(want_lse) and want_lse < 0:
                    assert np.all(out[t, h] == 0) and lse[t, h] == -math.inf, where
                    continue
                logit = np.concatenate([k["values"] @ x * scale for x, k in zip(queries, keys)])
                weights = np.exp(logit - want_lse)
                tol, tol_lse = bound(queries, keys, values, scale, want, weights)
                assert np.all(np.abs(out[t, h] - want) <= tol), (where, np.max(np.abs(out[t, h] - want) / tol))
                assert abs(lse[t, h] - want_lse) <= tol_lse + 2.0 ** -23 * abs(want_lse), (where, lse[t, h], want_lse)


def held_torch(x):
    """``held`` for many rows at once, fp64 on the rows' device."""
    x = x.double()
    lo, hi = x.min(-1).values, x.max(-1).values
    r = (15 / (hi - lo)).float().bfloat16().double()      # (rows of a range, whose two roundings do not meet a tie)
    return {"lo": lo, "step": 1 / r, "codes": torch.round((x - lo[..., None]) * r[..., None])}


def check_attend_torch(out, lse, q, k, v, seen, scale):
    """Rows of one batch against softmax attention in 64 bits, all at once: out, q [rows, d], k, v: ``held_torch`` of [rows or 1,
    keys, d] (keys padded), seen [rows]: how many of the keys a row sees.  The bound is that of ``bound``."""
    x = q.double()
    there = torch.arange(k["lo"].shape[1], device=x.device) < seen[:, None]
    parts = lambda a: (a["lo"], a["step"], a["codes"])
    (kl, ks, kc), (vl, vs, vc) = parts(k), parts(v)
    dot = lambda c, y: (c * y[:, None, :]).sum(-1)
    logit = (dot(kc, x) * ks + kl * x.sum(-1, keepdim=True)) * scale
    logit = torch.where(there, logit, -math.inf)
    want_lse = torch.logsumexp(logit, -1)
    some = seen > 0
    w = torch.where(there, torch.exp(logit - torch.where(some, want_lse, 0.0)[:, None]), 0.0)
    want = (w[..., None] * (vl[..., None] + vs[..., None] * vc)).sum(1)
    top = x.abs().max(-1, keepdim=True).values
    small = torch.where(x.abs() < 2.0 ** -7 * top, torch.minimum(2.0 ** -15 * top, 15 * x.abs()), 0.0).sum(-1, keepdim=True)
    cut = ks * (small + torch.where(small > 0, x.shape[1] / 16 * 2.0 ** -15 * top, 0.0))
    e = ((dot(kc, x.abs()) * ks + kl.abs() * x.abs().sum(-1, keepdim=True)) * (x.shape[1] + 12) * 2.0 ** -23 + cut) * scale
    e = torch.where(there, e, 0.0).max(-1).values
    mass = (w[..., None] * ((vl + 8 * vs).abs()[..., None] + vs[..., None] * (vc - 8).abs())).sum(1)
    ps = w * vs
    most = ps.max(-1).values
    cut = torch.minimum(2.0 ** -15 * most[:, None], 15 * ps).sum(-1) + 2.0 ** -12 * torch.minimum((seen / 64 + 2) * most, ps.sum(-1))
    rel = 2 * e + 2.0 ** -21 + (seen + 64) * 2.0 ** -23
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * rel)[:, None] * mass + (cut + 2.0 ** -20 * ps.sum(-1))[:, None] + 1e-37
    far = (out.double() - want).abs() > tol
    assert not far.any(), (far.any(-1).nonzero()[:5].tolist(), ((out.double() - want).abs() / tol).max().item())
    assert (lse[~some] == -math.inf).all()
    near = (lse.double() - want_lse).abs() <= e + 2.0 ** -20 + (seen + 64) * 2.0 ** -23 + 2.0 ** -23 * want_lse.abs()
    assert near[some].all(), (lse.double() - want_lse)[some].abs().max().item()
