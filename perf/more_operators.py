"""The operators between a projection and its attention in a multimodal step, as cases to time.

    rotate   queries and keys of each head are normalised and turned by their positions, which have one axis (text) or
             several (time, height, width of an image's or a video's patches)
    append   the same for keys on their way to the pages of a cache, their values beside them, queries to a tensor
    attend   a step's queries over that cache, where sequences of a batch share a prefix (many questions about one
             image or video): one softmax over the prefix's keys and the sequence's own

Where ``own`` is false the operators are computed in plain torch operations in 32 bits (the angles in 64), else by the
calls of ``paper_2602_01901_b200.paged``.

A pool holds one tensor (K or V) of one layer as bf16 [pages, kv_heads, page, head_dim]; a token's place is
(page id, token % page), its slot page id * page + token % page.  A row x of D elements becomes
y = x * rsqrt(mean(x^2) + eps) * w (where there is a norm), and then the pairs of its first ``rotary`` elements are turned:
pair i, elements (i, i + rotary / 2), or (2 i, 2 i + 1) where ``adjacent``, by positions[axis of i] * freqs[i].

Shapes are those of the repository's workloads (7B multi-head stacks of 32 heads, a grouped-query stack of 28 heads over 4,
images of 576 to 2 880 tokens, long video) and of its tests (64-wide heads), or generic.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6


def _rows_case(name, **fields):
    case = dict(op="rotate", tokens=1, spare=0, kv_heads=4, group=7, head_dim=128, rotary=128, axes=3, adjacent=False, norm=True,
                page=16, theta=1000000.0)
    case.update(fields)
    if name:
        case["name"] = name
    return case


def _attend_case(name, **fields):
    case = dict(op="attend", seqs=1, kv_heads=32, group=1, head_dim=128, page=16, low=1, high=1, groups=1, alone=0, pre_low=0,
                pre_high=0, queries=1, lazy=False, even=True)
    case.update(fields)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one user's next token on the grouped-query stack: latency
        _rows_case("rotate_token"),
        # an image's patches: two axes, neighbours as pairs, half of a 64-wide head turned, rows inside a fused projection
        _rows_case("rotate_patches_d64", tokens=1171, kv_heads=16, group=1, head_dim=64, rotary=32, axes=2, adjacent=True, theta=10000.0),
        # prompts of a batch on the multi-head stack
        _rows_case("rotate_prompts", tokens=16 * 675 + 13, kv_heads=32, group=1),
        # one token each of a batch of 32
        _rows_case("append_step_32", op="append", tokens=32),
        # an odd prompt chunk with padding behind it, 64-wide heads, no norm, one axis
        _rows_case("append_chunk_d64", op="append", tokens=1171, spare=109, kv_heads=16, group=1, head_dim=64, rotary=64, axes=1, norm=False,
                   page=32, theta=10000.0),
        # prompts of a batch on the multi-head stack: the most bytes
        _rows_case("append_prompts", op="append", tokens=16 * 675 + 13, kv_heads=32, group=1),
        # one user waiting for tokens about one image
        _attend_case("attend_single_user", low=131, high=131, pre_low=576, pre_high=576),
        # 32 questions about one image on the grouped-query stack, a lazy layer (the image's keys are scored by the Q Cache)
        _attend_case("attend_questions_32", seqs=32, kv_heads=4, group=7, low=40, high=352, pre_low=1024, pre_high=1024, lazy=True, even=False),
        # chats about five images and chats without any, multi-head stack, lengths far apart, one sequence without a token of its own
        _attend_case("attend_images_48", seqs=48, page=32, low=1, high=900, groups=5, alone=7, pre_low=576, pre_high=2880, even=False),
        # drafts of speculative decoding, 64-wide heads, one to five queries a sequence
        _attend_case("attend_drafts_d64", seqs=24, kv_heads=8, group=4, head_dim=64, low=30, high=1500, groups=3, alone=2, pre_low=2000,
                     pre_high=7000, queries=5, even=False),
        # long sequences that share nothing: the most bytes
        _attend_case("attend_own_long", seqs=8, low=8541, high=8541, groups=0),
        # a long video and 256 questions about it on the grouped-query stack: the most operations
        _attend_case("attend_video_256", seqs=256, kv_heads=4, group=7, page=64, low=20, high=200, pre_low=32768, pre_high=32768, even=False),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64])
    head_dim = rng.choice([64, 128, 128])
    if op != "attend":
        kv_heads, group = rng.choice([(1, 8), (2, 6), (4, 7), (8, 1), (8, 4), (16, 1), (32, 1), (3, 5)])
        tokens = _log(rng, 1, 1000000 // (kv_heads * (group + 2)))
        return _rows_case(None, op=op, tokens=tokens, spare=rng.choice([0, 0, rng.randint(1, 64)]) if op == "append" else 0, kv_heads=kv_heads,
                          group=group, head_dim=head_dim, rotary=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4]),
                          axes=rng.choice([1, 2, 3]), adjacent=rng.random() < 0.4, norm=rng.random() < 0.6, page=page,
                          theta=rng.choice([10000.0, 500000.0, 1000000.0]))
    while True:
        kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 7), (8, 1), (8, 4), (8, 8), (16, 1), (32, 1), (40, 1), (3, 5), (2, 16)])
        groups = rng.choice([0, 1, 1, 2, 4])
        seqs = _log(rng, max(1, groups), 256)
        high = _log(rng, 1, 9000)
        case = _attend_case(None, seqs=seqs, kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, high=high,
                            low=_log(rng, max(1, high // 20), high), groups=groups, alone=rng.randint(0, (seqs - groups) // 4) if groups else 0,
                            queries=rng.choice([1, 1, 1, 2, 5]), lazy=rng.random() < 0.4, even=rng.random() < 0.4)
        if groups:
            case["pre_high"] = _log(rng, 1, 32768)
            case["pre_low"] = _log(rng, max(1, case["pre_high"] // 10), case["pre_high"])
        w = work(case)
        if w["bytes"] <= 1.1e9 and w["flops"] <= 1.2e11 and seqs * high * kv_heads <= 2.2e6 and max(1, groups) * case["pre_high"] * kv_heads <= 2.2e6:
            return case


# ---- what a case's sizes are, from the case alone ----------------------------------------------------------

def _sizes(case):
    """(own lengths, with this step's tokens; queries of the sequences; where the groups begin and end; prefix lengths)."""
    rng = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    n, drafts, g = case["seqs"], max(1, case["queries"]), case["groups"]
    if case["even"]:
        lens, queries = [case["high"]] * n, [drafts] * n
    else:
        lens = [_log(rng, case["low"], case["high"]) for _ in range(n)]
        queries = [rng.randint(1, drafts) for _ in range(n)]
        if n > 2:                        # a sequence that stores nothing of its own, and one with a single token
            lens[rng.randrange(1, n)] = 1
            lens[0] = 0
    if g == 0:
        return lens, queries, [0], []
    first = rng.randint(0, case["alone"])                 # sequences without a prefix stand before and behind the groups
    last = n - (case["alone"] - first)
    cuts = sorted(rng.sample(range(first + 1, last), g - 1)) if g > 1 else []
    return lens, queries, [first] + cuts + [last], [_log(rng, case["pre_low"], case["pre_high"]) for _ in range(g)]


def work(case):
    if case["op"] != "attend":
        total, heads = case["tokens"] + case["spare"], case["kv_heads"] * case["group"]
        rows = total * (heads + case["kv_heads"]) + (case["kv_heads"] * case["tokens"] if case["op"] == "append" else 0)
        if case["op"] == "append":
            rows -= case["spare"] * case["kv_heads"]       # rows of no slot are not stored
        return {"bytes": 4.0 * rows * case["head_dim"] + 4.0 * total * (case["axes"] + (case["op"] == "append")), "flops": 6.0 * rows * case["head_dim"]}
    lens, queries, groups, pre = _sizes(case)
    heads, d = case["kv_heads"] * case["group"], case["head_dim"]
    tokens = sum(lens) + sum(pre)
    pairs = sum(n * q for n, q in zip(lens, queries)) + sum(p * sum(queries[a:b]) for p, a, b in zip(pre, groups, groups[1:]))
    rows = sum(queries) * heads
    return {"bytes": 4.0 * tokens * case["kv_heads"] * d + rows * d * 2.0 * (3 if case["lazy"] and pre else 2) + 4.0 * rows, "flops": 4.0 * pairs * heads * d}


# ---- inputs --------------------------------------------------------------------------------------------------

def _rows(shape, gen):
    """Rows as projections give them: some channels larger than others, tokens of different size."""
    channel = torch.exp(0.5 * torch.randn(shape[1:], device=DEVICE, generator=gen))
    token = torch.exp(0.3 * torch.randn((shape[0],) + (1,) * (len(shape) - 1), device=DEVICE, generator=gen))
    return (torch.randn(shape, device=DEVICE, generator=gen) * channel * token).bfloat16()


def _table_of(lens, page, rows, ids, gen):
    """Scattered pages of sequences of given lengths, in the table rows that they have: (pages, lens, number of pages)."""
    n_pages = sum(-(-n // page) for n in lens) + 3
    max_pages = max(1, max([-(-n // page) for n in lens] + [0]) + 2)
    order = torch.randperm(n_pages, device=DEVICE, generator=gen).to(torch.int32)
    held = torch.tensor([-(-n // page) for n in lens], device=DEVICE)
    first = torch.cumsum(held, 0) - held
    col = torch.arange(max_pages, device=DEVICE)
    at = (first[:, None] + col).clamp_(max=n_pages - 1)
    pages = torch.full((rows, max_pages), -1, dtype=torch.int32, device=DEVICE)
    pages[ids.long()] = torch.where(col < held[:, None], order[at], -1)
    long = torch.zeros(rows, dtype=torch.int32, device=DEVICE)
    long[ids.long()] = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    return pages, long, n_pages


def _stream(case, lens, rows, ids, gen):
    page, heads, d = case["page"], case["kv_heads"], case["head_dim"]
    pages, long, n_pages = _table_of(lens, page, rows, ids, gen)
    live = torch.zeros(n_pages, page, dtype=torch.bool, device=DEVICE)
    used = torch.arange(pages.shape[1] * page, device=DEVICE).reshape(1, -1, page) < long[:, None, None]
    live.view(-1)[(pages.clamp(min=0).long()[..., None] * page + torch.arange(page, device=DEVICE))[used]] = True
    pools = []
    for _ in "kv":
        rows_of = _rows((n_pages * page, heads, d), gen).reshape(n_pages, page, heads, d)
        rows_of[~live] = math.nan                          # what stands where no token is
        pools.append(rows_of.transpose(1, 2).contiguous())
    return {"k_pool": pools[0], "v_pool": pools[1], "pages": pages, "lens": long}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 2 + 1)
    randint = lambda low, high, shape: torch.randint(low, high, shape, device=DEVICE, generator=gen)
    if case["op"] != "attend":
        n, total, heads, d, page = case["tokens"], case["tokens"] + case["spare"], case["kv_heads"], case["head_dim"], case["page"]
        q_heads, half = heads * case["group"], case["rotary"] // 2
        fused = _rows((total, q_heads + 2 * heads, d), gen)             # a fused projection's output: q, k, v
        # text runs on from far behind; an image's or a video's patches count rows and columns from where they begin
        width = 1 + int(randint(8, 60, (1,)))
        i, base = torch.arange(total, device=DEVICE), randint(0, 130000, (1,))
        axes = [base + i // (width * width), base + i // width % width, base + i % width]
        positions = torch.stack((axes if case["axes"] == 3 else axes[1:] if case["axes"] == 2 else [base + i])).to(torch.int32)
        freqs = (case["theta"] ** (-torch.arange(half, dtype=torch.float64) / half)).float()
        axis = [j * case["axes"] // half for j in range(half)]
        state = {"case": dict(case), "q": fused[:, :q_heads], "k": fused[:, q_heads:q_heads + heads], "positions": positions,
                 "freqs": freqs.to(DEVICE), "axes": torch.tensor(axis, dtype=torch.int32, device=DEVICE), "norms": None}
        if case["norm"]:
            state["norms"] = tuple((1 + 0.2 * torch.randn(d, device=DEVICE, generator=gen)).bfloat16() for _ in "qk")
        if case["op"] == "append":
            n_pages = -(-n // page) + 2
            if n <= 64:                  # single tokens of a batch: each in a page of its sequence's own
                n_pages = n + 2
                slots = torch.randperm(n_pages, device=DEVICE, generator=gen)[:n] * page + randint(0, page, (n,))
            else:                        # prompts lie in their pages token by token
                order = torch.randperm(n_pages, device=DEVICE, generator=gen)
                j = torch.arange(n, device=DEVICE) + int(randint(0, page, (1,)))
                slots = order[j // page] * page + j % page
            state["slots"] = torch.cat([slots, torch.full((case["spare"],), -1, device=DEVICE)]).to(torch.int32)
            state["v"] = fused[:, q_heads + heads:]
            state["k_pool"], state["v_pool"] = (torch.zeros(n_pages, heads, page, d, dtype=torch.bfloat16, device=DEVICE) for _ in "kv")
        return state
    lens, queries, groups, pre = _sizes(case)
    n, heads, d = case["seqs"], case["kv_heads"] * case["group"], case["head_dim"]
    ids = torch.randperm(n + 3, device=DEVICE, generator=gen)[:n].to(torch.int32)
    q = lambda: torch.randn(sum(queries), heads, d, device=DEVICE, generator=gen).bfloat16()
    state = {"case": dict(case), "ids": ids, "starts": torch.tensor([0] + queries, device=DEVICE).cumsum(0).to(torch.int32), "most": max(queries),
             "q": q(), "own": _stream(case, lens, n + 3, ids, gen)}
    if pre:
        state["shared_ids"] = torch.randperm(len(pre) + 2, device=DEVICE, generator=gen)[:len(pre)].to(torch.int32)
        state["groups"] = torch.tensor(groups, dtype=torch.int32, device=DEVICE)
        state["shared"] = _stream(case, pre, len(pre) + 2, state["shared_ids"], gen)
        state["q_shared"] = q() if case["lazy"] else state["q"]          # a lazy layer's: the Q Cache
        state["most_shared"] = max(sum(queries[a:b]) for a, b in zip(groups, groups[1:]))
    return state


# ---- the passes ----------------------------------------------------------------------------------------------

def _turned(x, norm, cos, sin, case):
    """bf16 rows [tokens, heads, d] -> their norm and rotation, fp32."""
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * norm.float()
    r = case["rotary"]
    part, rest = x[..., :r], x[..., r:]
    a, b = (part[..., 0::2], part[..., 1::2]) if case["adjacent"] else (part[..., :r // 2], part[..., r // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if case["adjacent"] else torch.cat([u, v], -1), rest], -1)


def _rotate(s):
    case, (q_norm, k_norm) = s["case"], s["norms"] or (None, None)
    if own:
        from paper_2602_01901_b200 import paged

        rotation = paged.Rotation(s["freqs"], s["axes"], case["adjacent"])
        if case["op"] == "rotate":
            return paged.rotate(s["q"], s["k"], s["positions"], rotation, q_norm=q_norm, k_norm=k_norm, eps=EPS)
        q = paged.append(s["k_pool"], s["v_pool"], s["slots"], s["k"], s["v"], q=s["q"], positions=s["positions"], rotation=rotation, q_norm=q_norm,
                         k_norm=k_norm, eps=EPS)
        return q, s["k_pool"], s["v_pool"]
    angle = s["positions"].double()[s["axes"].long()].T * s["freqs"].double()          # [tokens, pairs]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    q, k = (_turned(x, norm, cos, sin, case).bfloat16() for x, norm in ((s["q"], q_norm), (s["k"], k_norm)))
    if case["op"] == "rotate":
        return q, k
    there = s["slots"] >= 0
    page, place = s["slots"][there].long() // case["page"], s["slots"][there].long() % case["page"]
    s["k_pool"][page, :, place] = k[there]
    s["v_pool"][page, :, place] = s["v"][there]
    return q, s["k_pool"], s["v_pool"]


def _part(q, t, rows, last, case):
    """Softmax sums over one stream: q [n, queries, heads, d] of table rows ``rows``, each query seeing ``last`` [n, queries] keys.
    Returns (largest score, sum, weighted values), [n, queries, heads(, d)]."""
    n, most, d = q.shape[0], q.shape[1], case["head_dim"]
    heads, group = case["kv_heads"], case["group"]
    ids = t["pages"][rows].clamp(min=0).long()
    key = torch.arange(ids.shape[1] * case["page"], device=ids.device)
    seen = (key < t["lens"][rows][:, None])[:, None, :, None]
    k, v = (torch.where(seen, t[x][ids].float().permute(0, 2, 1, 3, 4).flatten(2, 3), 0.0) for x in ("k_pool", "v_pool"))   # [n, heads, keys, d]
    q = q.float().reshape(n, most, heads, group, d).transpose(1, 2).reshape(n, heads, most * group, d)
    score = (q @ k.transpose(2, 3) / math.sqrt(d)).reshape(n, heads, most, group, -1)
    score = score.masked_fill((key >= last[..., None])[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top.isfinite(), top, 0.0))
    values = (weight.reshape(n, heads, most * group, -1) @ v).reshape(n, heads, most, group, d)
    out = lambda x: x.transpose(1, 2).reshape(n, most, heads * group, *x.shape[4:])
    return out(top[..., 0]), out(weight.sum(-1)), out(values)


def _attend(s):
    case = s["case"]
    if own:
        from paper_2602_01901_b200 import paged

        t, p = s["own"], s.get("shared")
        shared = paged.Stream(s["q_shared"], p["k_pool"], p["v_pool"], p["pages"], p["lens"]) if p else None
        return paged.attend(paged.Stream(s["q"], t["k_pool"], t["v_pool"], t["pages"], t["lens"]), shared=shared, groups=s.get("groups"),
                            shared_ids=s.get("shared_ids"), seq_ids=s["ids"], starts=s["starts"], max_queries=s["most"])
    starts, rows = s["starts"].long(), s["ids"].long()
    tokens, heads, d, most = s["q"].shape[0], s["q"].shape[1], case["head_dim"], s["most"]
    count = starts[1:] - starts[:-1]
    place = torch.arange(most, device=starts.device)
    at = (starts[:-1, None] + place).clamp_(max=tokens - 1)
    # the own tokens end with the queries': a query sees what is not behind it
    last = (s["own"]["lens"][rows][:, None] - (count[:, None] - 1 - place)).clamp_(min=0)
    parts = [(torch.where(place < count[:, None], at, tokens), _part(s["q"][at], s["own"], rows, last, case))]
    if "shared" in s:
        begin = starts[s["groups"].long()]
        count = begin[1:] - begin[:-1]
        place = torch.arange(s["most_shared"], device=starts.device)
        at = (begin[:-1, None] + place).clamp_(max=tokens - 1)
        rows = s["shared_ids"].long()
        last = s["shared"]["lens"][rows][:, None].expand(-1, len(place))
        parts.append((torch.where(place < count[:, None], at, tokens), _part(s["q_shared"][at], s["shared"], rows, last, case)))
    # both parts token by token (padded queries go to a row of their own behind the last), then as one softmax
    tops, sums, values = [], [], []
    for to, (top, total, value) in parts:
        tops.append(torch.full((tokens + 1, heads), -math.inf, device=to.device).index_put_((to,), top)[:-1])
        sums.append(torch.zeros(tokens + 1, heads, device=to.device).index_put_((to,), total)[:-1])
        values.append(torch.zeros(tokens + 1, heads, d, device=to.device).index_put_((to,), value)[:-1])
    tops, sums, values = torch.stack(tops), torch.stack(sums), torch.stack(values)
    top = tops.amax(0)
    scale = torch.exp(tops - torch.where(top.isfinite(), top, 0.0))
    total = (sums * scale).sum(0)
    out = (values * scale[..., None]).sum(0) / torch.where(total > 0, total, 1.0)[..., None]
    return out.bfloat16(), torch.where(total > 0, top + torch.log(total), -math.inf)


def run(state):
    return _attend(state) if state["case"]["op"] == "attend" else _rotate(state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------

def _exact_rows(x, norm, s):
    """Element by element: what an element's partner is, its sign and its pair."""
    case = s["case"]
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["head_dim"] + EPS) * norm.double()
    e = torch.arange(case["rotary"], device=x.device)
    half = case["rotary"] // 2
    partner, pair, second = (e ^ 1, e // 2, e % 2 == 1) if case["adjacent"] else ((e + half) % case["rotary"], e % half, e >= half)
    axes, freqs = s["axes"].tolist(), s["freqs"].tolist()
    angle = torch.stack([s["positions"][axes[p]].double() * freqs[p] for p in pair.tolist()], -1)[:, None]
    turned = x[..., :case["rotary"]] * torch.cos(angle) + torch.where(second, 1.0, -1.0) * x[..., partner] * torch.sin(angle)
    return torch.cat([turned, x[..., case["rotary"]:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] != "attend":
        q_norm, k_norm = s["norms"] or (None, None)
        q, k = _exact_rows(s["q"], q_norm, s), _exact_rows(s["k"], k_norm, s)
        if case["op"] == "rotate":
            return q, k
        found = [q]
        for rows, pool in ((k, s["k_pool"]), (s["v"].double(), s["v_pool"])):
            flat = pool.double().transpose(1, 2).flatten(0, 1)          # by slot
            flat[s["slots"][:case["tokens"]].long()] = rows[:case["tokens"]]
            found.append(flat.reshape(pool.shape[0], case["page"], case["kv_heads"], case["head_dim"]).transpose(1, 2))
        return tuple(found)
    lens, queries, groups, pre = _sizes(case)
    page, d, group = case["page"], case["head_dim"], case["group"]
    begin = s["starts"].tolist()
    of = {i: g for g in range(len(pre)) for i in range(groups[g], groups[g + 1])}

    def rows_of(t, row, length, head):
        pos = torch.arange(length, device=DEVICE)
        ids = t["pages"][row].long()[pos // page]
        return t["k_pool"][ids, head, pos % page].double(), t["v_pool"][ids, head, pos % page].double()

    out = torch.zeros(begin[-1], case["kv_heads"] * group, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((begin[-1], case["kv_heads"] * group), -math.inf, dtype=torch.float64, device=DEVICE)
    rows, shared_rows = s["ids"].tolist(), s["shared_ids"].tolist() if pre else []
    for h in range(case["kv_heads"]):
        cols = slice(h * group, (h + 1) * group)
        held = [rows_of(s["shared"], shared_rows[g], n, h) for g, n in enumerate(pre)]
        for i, n in enumerate(lens):
            a, b = begin[i], begin[i + 1]
            k, v = rows_of(s["own"], rows[i], n, h)
            logit = torch.einsum("qgd,ld->qgl", s["q"][a:b, cols].double(), k) / math.sqrt(d)
            behind = torch.arange(n, device=DEVICE)[None] > (n - (b - a) + torch.arange(b - a, device=DEVICE))[:, None]
            logit = torch.where(behind[:, None], -math.inf, logit)
            if i in of:
                kp, vp = held[of[i]]
                logit = torch.cat([torch.einsum("qgd,ld->qgl", s["q_shared"][a:b, cols].double(), kp) / math.sqrt(d), logit], -1)
                v = torch.cat([vp, v])
            if logit.shape[-1] == 0:
                continue
            total = torch.logsumexp(logit, -1)
            weight = torch.where(total[..., None].isfinite(), torch.exp(logit - total[..., None]), 0.0)
            out[a:b, cols], lse[a:b, cols] = weight @ v, total
    return out, lse
