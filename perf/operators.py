"""The operators around a K/V cache that is held in 4 bits, as cases to time.

A program that serves long multimodal prompts keeps its cache in 4 bits, in pages, and does three things
with it in every step:

    tables   the page tables of the batch are made longer by each sequence's new tokens and shorter by the
             tokens (drafts that were turned down, finished sequences) that leave, and every new token gets
             the place ("slot") where its rows go
    append   the new tokens' K and V rows are quantised and stored at their slots, and read back as the values
             that later steps will see (what the attention inside a prompt chunk is computed on)
    attend   the new tokens' queries attend over everything that is cached, in one stream or in a text and a
             visual stream with a query each (an ordinary layer, or a lazy one)

Where ``own`` is false the operators are computed in plain torch operations in 32 bits, straight from the
format of the pages, which is:

    A pool holds one tensor (K or V) of one layer and stream: ``pages`` pages of ``page`` tokens, each page
    first the codes [kv_heads][page / 16][8 * head_dim bytes] and then the parameters [kv_heads][page] of 4 bytes.
    A row (one token, one head) is quantised as a whole: lo = its smallest value, r = bf16(15 / (largest - lo)),
    code = round((x - lo) * r) in 0..15; it stands for lo + code / r, or lo where r is 0 (a range below 2^-100).
    Parameters: lo as bf16 in the low half, r as bf16 in the high half.
    Codes of a block of 16 tokens, in bytes of two, the first one in the low half:
        K, 128 wide  [token % 2][token / 2][d / 32][d / 2 % 16]
        K,  64 wide  [token / 2][d / 16][token % 2][d / 2 % 8]
        V, 128 wide  [d / 8 % 2][d / 16][token / 4][d / 2 % 4][token % 4]
        V,  64 wide  [d / 8][token / 4][d / 2 % 4][token % 4]

Shapes are those of the repository's workloads (7B multi-head stacks, a grouped-query stack of 28 heads over 4,
image prompts of 576 to 2 880 visual tokens, long pruned video) or generic ones.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
NAN_PARAMS = 0x7FC07FC0          # what stands in the parameters of rows that no token has


def _case(name, **fields):
    case = dict(op="attend", seqs=1, kv_heads=32, group=1, head_dim=128, page=16, low=1, high=1, vis_low=0, vis_high=0,
                queries=1, even=True, spare=0)
    case.update(fields)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a small batch takes one token each: what a step's bookkeeping costs
        _case("tables_step_8", op="tables", seqs=8, low=700, high=1100, page=16),
        # speculative decoding of a large batch: one to eight drafts each, all turned down again
        _case("tables_drafts_256", op="tables", seqs=256, low=90, high=6000, page=16, queries=8, even=False),
        # a batch of finished sequences leaves and one with long prompts enters
        _case("tables_prompts_64", op="tables", seqs=64, low=500, high=9000, page=32, queries=0, even=False),
        # one token each of a batch on the grouped-query stack
        _case("append_step_32", op="append", seqs=32, kv_heads=4, group=7),
        # an odd prompt chunk with padding behind it, 64-wide heads, rows inside a fused projection's output
        _case("append_chunk_d64", op="append", seqs=1171, kv_heads=16, head_dim=64, page=32, spare=109),
        # prompts of a batch on the multi-head stack
        _case("append_prompts", op="append", seqs=16 * 675 + 13, kv_heads=32),
        # one user waiting for tokens: short image prompt, text and visual stream
        _case("attend_single_user", low=131, high=131, vis_low=576, vis_high=576),
        # grouped-query stack, large batch, text and visual stream
        _case("attend_gqa_32", seqs=32, kv_heads=4, group=7, low=100, high=352, vis_low=1024, vis_high=1024, even=False),
        # multi-head stack, batch of 16, lengths far apart, one sequence empty and one of a single token
        _case("attend_ragged_16", seqs=16, kv_heads=32, low=60, high=5000, page=32, even=False),
        # drafts of speculative decoding, 64-wide heads, one to five queries a sequence
        _case("attend_drafts_d64", seqs=24, kv_heads=8, group=4, head_dim=64, low=300, high=7000, queries=5, even=False),
        # few sequences, very long text
        _case("attend_long_gqa", seqs=3, kv_heads=8, group=4, low=90001, high=90001, page=64),
        # high-resolution images and long video on the multi-head stack: the most bytes
        _case("attend_mha_video", seqs=8, kv_heads=32, low=349, high=349, vis_low=8192, vis_high=8192),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64])
    if op == "tables":
        high = _log(rng, 20, 9000)
        return _case(None, op=op, seqs=_log(rng, 1, 256 if high > 2000 else 1024), page=page, low=_log(rng, 1, high), high=high,
                     queries=rng.choice([0, 1, 1, 3, 8]), even=rng.random() < 0.3)
    head_dim = rng.choice([64, 128, 128])
    if op == "append":
        kv_heads = rng.choice([1, 2, 4, 8, 16, 32])
        rows = _log(rng, 1, 340000)
        tokens = max(1, rows // kv_heads)
        return _case(None, op=op, seqs=tokens, kv_heads=kv_heads, group=rng.choice([1, 4, 7]), head_dim=head_dim, page=page,
                     spare=rng.choice([0, 0, rng.randint(1, 64)]))
    while True:
        kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 7), (8, 1), (8, 4), (8, 8), (16, 1), (32, 1), (40, 1), (3, 5), (2, 16)])
        high = _log(rng, 1, 90000)
        case = _case(None, op=op, seqs=_log(rng, 1, 64), kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, high=high,
                     low=_log(rng, max(1, high // 20), high), queries=rng.choice([1, 1, 1, 2, 5]), even=rng.random() < 0.4)
        if rng.random() < 0.4:
            case["vis_high"] = _log(rng, 1, 9000)
            case["vis_low"] = _log(rng, max(1, case["vis_high"] // 10), case["vis_high"])
        if work(case)["bytes"] <= 2.9e8 and case["seqs"] * (high + case["vis_high"]) * kv_heads <= 2.2e6:
            return case


# ---- what a case's sizes are, from the case alone ----------------------------------------------------------

def _sizes(case):
    """(text lengths, visual lengths, queries) of the sequences, after this step's tokens have been stored."""
    rng = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    n, drafts = case["seqs"], max(1, case["queries"])
    if case["even"]:
        return [case["high"]] * n, [case["vis_high"]] * n, [drafts] * n
    text = [_log(rng, case["low"], case["high"]) for _ in range(n)]
    vis = [_log(rng, case["vis_low"], case["vis_high"]) if case["vis_high"] else 0 for _ in range(n)]
    queries = [rng.randint(1, drafts) for _ in range(n)]
    if n > 2:                        # a sequence with nothing yet, and one with a single token
        text[rng.randrange(1, n)] = 1
        text[0] = vis[0] = 0
    return text, vis, queries


def _page_bytes(case):
    return case["kv_heads"] * case["page"] * (case["head_dim"] // 2 + 4)


def work(case):
    if case["op"] == "tables":
        text, _, queries = _sizes(case)
        new = text if case["queries"] == 0 else queries
        pages = sum(-(-(t + (0 if case["queries"] == 0 else q)) // case["page"]) - (0 if case["queries"] == 0 else -(-t // case["page"]))
                    for t, q in zip(text, new))
        # lengths in and out, a slot per new token; a page that is taken is read from the free pages and written to its
        # table, and one that leaves the same the other way
        return {"bytes": 4.0 * (4 * len(text) + sum(new) + 4 * pages), "flops": 0.0}
    row = case["head_dim"] // 2 + 4
    if case["op"] == "append":
        rows = 2.0 * case["seqs"] * case["kv_heads"]
        return {"bytes": rows * (2 * 2 * case["head_dim"] + row) + 4.0 * (case["seqs"] + case["spare"]), "flops": 6.0 * rows * case["head_dim"]}
    text, vis, queries = _sizes(case)
    heads = case["kv_heads"] * case["group"]
    tokens = sum(t + v for t, v in zip(text, vis))
    pairs = sum(q * (t + v) for t, v, q in zip(text, vis, queries))
    q_rows = sum(queries) * heads
    q_reads = 2 if case["vis_high"] else 1
    return {"bytes": 2.0 * tokens * case["kv_heads"] * row + q_rows * case["head_dim"] * 2.0 * (1 + q_reads) + 4.0 * q_rows,
            "flops": 4.0 * pairs * heads * case["head_dim"]}


# ---- the format, in torch ------------------------------------------------------------------------------------

def _quantise(x):
    """bf16 [..., head_dim] -> codes uint8 of the same shape, parameters int32 [...]."""
    lo, hi = x.amin(-1).float(), x.amax(-1).float()
    span = hi - lo
    r = torch.where(span >= 2.0 ** -100, 15.0 / span, torch.zeros_like(span)).bfloat16()
    codes = torch.round((x.float() - lo[..., None]) * r.float()[..., None]).clamp_(0, 15).to(torch.uint8)
    bits = lambda t: t.bfloat16().view(torch.int16).to(torch.int32) & 0xFFFF
    return codes, bits(lo) | (bits(r) << 16)


#: the axes of a block's bytes (with the two halves of a byte last), and how [token, d] is put together from them
_AXES = {("k", 128): ((2, 8, 4, 16, 2), (1, 0, 2, 3, 4)), ("k", 64): ((8, 4, 2, 8, 2), (0, 2, 1, 3, 4)),
         ("v", 128): ((2, 8, 4, 4, 4, 2), (2, 4, 1, 0, 3, 5)), ("v", 64): ((8, 4, 4, 4, 2), (1, 3, 0, 2, 4))}


def _to_bytes(codes, which):
    """codes [..., 16, head_dim] of whole blocks -> their bytes [..., 8 * head_dim]."""
    shape, order = _AXES[which, codes.shape[-1]]
    lead = codes.dim() - 2
    back = [order.index(i) for i in range(len(order))]
    x = codes.reshape(*codes.shape[:-2], *[shape[i] for i in order]).permute(*range(lead), *[lead + i for i in back])
    return (x[..., 0] | (x[..., 1] << 4)).reshape(*codes.shape[:-2], -1)


def _to_codes(raw, which, head_dim):
    """The inverse of ``_to_bytes``."""
    shape, order = _AXES[which, head_dim]
    lead = raw.dim() - 1
    x = torch.stack([raw & 15, raw >> 4], -1).reshape(*raw.shape[:-1], *shape)
    return x.permute(*range(lead), *[lead + i for i in order]).reshape(*raw.shape[:-1], 16, head_dim)


def _pages_of(codes, params, which):
    """codes [pages, page, heads, head_dim], params [pages, page, heads] -> the pool's bytes [pages, page bytes]."""
    n, page, heads, head_dim = codes.shape
    blocks = codes.permute(0, 2, 1, 3).reshape(n, heads, page // 16, 16, head_dim)
    words = params.permute(0, 2, 1).contiguous().reshape(n, -1)
    return torch.cat([_to_bytes(blocks, which).reshape(n, -1), words.view(torch.uint8)], 1)


def _values(raw, case, which):
    """Bytes [..., page bytes] of pages -> what they stand for, fp32 [..., page, heads, head_dim]."""
    heads, page, head_dim = case["kv_heads"], case["page"], case["head_dim"]
    lead, n = raw.shape[:-1], heads * page * head_dim // 2
    codes = _to_codes(raw[..., :n].reshape(*lead, heads, page // 16, 8 * head_dim), which, head_dim).reshape(*lead, heads, page, head_dim)
    words = raw[..., n:].contiguous().view(torch.int32).reshape(*lead, heads, page)
    lo, r = (words << 16).view(torch.float32), (words & -65536).view(torch.float32)
    step = torch.where(r > 0, 1.0 / r, torch.zeros_like(r))
    return (lo[..., None] + codes.float() * step[..., None]).transpose(-3, -2)


# ---- inputs --------------------------------------------------------------------------------------------------

def _rows(shape, gen):
    """K/V rows as projections give them: some channels larger than others, tokens of different size."""
    channel = torch.exp(0.5 * torch.randn(shape[1:], device=DEVICE, generator=gen))
    token = torch.exp(0.3 * torch.randn((shape[0],) + (1,) * (len(shape) - 1), device=DEVICE, generator=gen))
    return (torch.randn(shape, device=DEVICE, generator=gen) * channel * token).bfloat16()


def _table_of(lens, n_pages, page, rows, ids, gen):
    """Scattered pages of sequences of given lengths, in the table rows that they have: (pages, lens, free, state)."""
    max_pages = max(1, max(-(-n // page) for n in lens) + 2)
    order = torch.randperm(n_pages, device=DEVICE, generator=gen).to(torch.int32)
    held = torch.tensor([-(-n // page) for n in lens], device=DEVICE)
    first = torch.cumsum(held, 0) - held
    col = torch.arange(max_pages, device=DEVICE)
    at = (first[:, None] + col).clamp_(max=n_pages - 1)
    pages = torch.full((rows, max_pages), -1, dtype=torch.int32, device=DEVICE)
    pages[ids.long()] = torch.where(col < held[:, None], order[at], -1)
    long = torch.zeros(rows, dtype=torch.int32, device=DEVICE)
    long[ids.long()] = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    used = sum(-(-n // page) for n in lens)
    free = torch.cat([order[used:].flip(0), order[:used].flip(0)]).contiguous()   # the first free page is the last of them
    state = torch.tensor([n_pages - used, 0, 0, 0], dtype=torch.int32, device=DEVICE)
    return pages, long, free, state


def _stream(case, lens, rows, ids, gen):
    page, heads, head_dim = case["page"], case["kv_heads"], case["head_dim"]
    n_pages = sum(-(-n // page) for n in lens) + 3
    pages, long, _, _ = _table_of(lens, n_pages, page, rows, ids, gen)
    live = torch.zeros(n_pages, page, dtype=torch.bool, device=DEVICE)
    used = torch.arange(pages.shape[1] * page, device=DEVICE).reshape(1, -1, page) < long[:, None, None]
    at = pages.clamp(min=0).long()[..., None] * page + torch.arange(page, device=DEVICE)
    live.view(-1)[at[used]] = True
    pools = []
    for which in "kv":
        out = torch.empty(n_pages, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
        step = max(1, (1 << 26) // (page * heads * head_dim))
        for a in range(0, n_pages, step):
            b = min(n_pages, a + step)
            codes, params = _quantise(_rows(((b - a) * page, heads, head_dim), gen).reshape(b - a, page, heads, head_dim))
            params = torch.where(live[a:b, :, None], params, NAN_PARAMS)
            out[a:b] = _pages_of(codes, params, which)
        pools.append(out)
    return {"k_pool": pools[0], "v_pool": pools[1], "pages": pages, "lens": long}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 2 + 1)
    text, vis, queries = _sizes(case)
    n = case["seqs"]
    if case["op"] == "append":
        heads, head_dim, page = case["kv_heads"], case["head_dim"], case["page"]
        q_heads, total = heads * case["group"], n + case["spare"]
        fused = _rows((total, q_heads + 2 * heads, head_dim), gen)          # a fused projection's output: q, k, v
        n_pages = -(-n // page) + 2
        # prompts lie in their pages token by token; a batch's single tokens each in a page of their sequence's own
        if n <= 64:
            n_pages = n + 2
            slots = torch.randperm(n_pages, device=DEVICE, generator=gen)[:n] * page + torch.randint(0, page, (n,), device=DEVICE, generator=gen)
        else:
            order = torch.randperm(n_pages, device=DEVICE, generator=gen)
            i = torch.arange(n, device=DEVICE) + int(torch.randint(0, page, (1,), device=DEVICE, generator=gen))
            slots = order[i // page] * page + i % page
        slots = torch.cat([slots, torch.full((case["spare"],), -1, device=DEVICE)]).to(torch.int32)
        pool = lambda: torch.zeros(n_pages, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
        back = lambda: torch.zeros(total, heads, head_dim, dtype=torch.bfloat16, device=DEVICE)
        return {"case": dict(case), "k": fused[:, q_heads:q_heads + heads], "v": fused[:, q_heads + heads:], "slots": slots,
                "k_pool": pool(), "v_pool": pool(), "k_back": back(), "v_back": back()}
    rows = n + 3
    ids = torch.randperm(rows, device=DEVICE, generator=gen)[:n].to(torch.int32)
    if case["op"] == "tables":
        page = case["page"]
        new = text if case["queries"] == 0 else queries
        room = 2 * sum(-(-(t + q) // page) for t, q in zip(text, new)) + 7
        pages, lens, free, state = _table_of(text, room, page, rows, ids, gen)
        grown = torch.zeros(rows, max(-(-(t + q) // page) for t, q in zip(text, new)) + 1, dtype=torch.int32, device=DEVICE) - 1
        width = min(grown.shape[1], pages.shape[1])
        grown[:, :width] = pages[:, :width]
        new = torch.tensor(new, dtype=torch.int32, device=DEVICE)
        if case["queries"] == 0:      # the next batch's prompts: the same sizes in another order
            new = new[torch.randperm(n, device=DEVICE, generator=gen)].contiguous()
        return {"case": dict(case), "pages": grown, "lens": lens, "free": free, "state": state, "ids": ids, "new": new,
                "keep": lens[ids.long()].contiguous(), "most": sum(text if case["queries"] == 0 else queries) + 5}
    starts = torch.tensor([0] + queries, device=DEVICE).cumsum(0).to(torch.int32)
    heads, total = case["kv_heads"] * case["group"], sum(queries)
    state = {"case": dict(case), "ids": ids, "starts": starts, "most": max(queries),
             "q": torch.randn(total, heads, case["head_dim"], device=DEVICE, generator=gen).bfloat16(),
             "text": _stream(case, text, rows, ids, gen)}
    if case["vis_high"]:              # the visual keys are scored by the Q Cache, the leader's queries
        state["q_visual"] = torch.randn(total, heads, case["head_dim"], device=DEVICE, generator=gen).bfloat16()
        state["visual"] = _stream(case, vis, rows, ids, gen)
    return state


# ---- the passes ----------------------------------------------------------------------------------------------

def _tables(s):
    page, pages, lens, free, state, ids = s["case"]["page"], s["pages"], s["lens"], s["free"], s["state"], s["ids"]
    prompts = s["case"]["queries"] == 0
    if own:
        from paper_2602_01901_b200 import quant

        table = quant.PageTable(pages, lens, free, state, page)
        if prompts:
            quant.table_trim(table, None, seq_ids=ids)
        starts, slots = quant.table_extend(table, s["new"], seq_ids=ids, max_slots=s["most"])
        if not prompts:
            quant.table_trim(table, s["keep"], seq_ids=ids)
    else:
        rows = ids.long()
        if prompts:
            _trim(page, pages, lens, free, state, rows, torch.zeros_like(s["keep"]))
        starts, slots = _extend(page, pages, lens, free, state, rows, s["new"], s["most"])
        if not prompts:
            _trim(page, pages, lens, free, state, rows, s["keep"])
    return {"starts": starts, "slots": slots, "pages": pages, "lens": lens, "free": free, "state": state}


def _extend(page, pages, lens, free, state, rows, new, most):
    """Sequence after sequence, page after page: the next page is the last one of the free ones."""
    old = lens[rows]
    have, want = (old + page - 1) // page, (old + new + page - 1) // page
    first = torch.cumsum(want - have, 0) - (want - have)
    col = torch.arange(pages.shape[1], device=pages.device)
    taken = (col >= have[:, None]) & (col < want[:, None])
    at = (state[0] - 1 - (first[:, None] + col - have[:, None])).clamp(0, free.numel() - 1)
    pages[rows] = torch.where(taken, free[at], pages[rows])
    starts = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0).to(torch.int32)])
    i = torch.arange(most, device=pages.device, dtype=torch.int32)
    seq = torch.searchsorted(starts[1:].contiguous(), i, right=True).clamp_(max=len(rows) - 1)
    pos = old[seq] + i - starts[seq]
    place = pages[rows[seq], (pos // page).clamp(0, pages.shape[1] - 1).long()] * page + pos % page
    slots = torch.where(i < starts[-1], place, -1).to(torch.int32)
    lens[rows] = old + new
    state[0] -= (want - have).sum()
    return starts, slots


def _trim(page, pages, lens, free, state, rows, keep):
    """The inverse: what is given back is taken again in the same order."""
    old = lens[rows]
    left = torch.minimum(old, keep)
    have, want = (old + page - 1) // page, (left + page - 1) // page
    first = torch.cumsum(have - want, 0) - (have - want)
    col = torch.arange(pages.shape[1], device=pages.device)
    given = (col >= want[:, None]) & (col < have[:, None])
    total = (have - want).sum()
    at = torch.where(given, state[0] + total - 1 - (first[:, None] + col - want[:, None]), free.numel())
    longer = torch.cat([free, free[:1]])
    longer[at] = pages[rows]
    free.copy_(longer[:-1])
    pages[rows] = torch.where(given, -1, pages[rows])
    lens[rows] = left
    state[0] += total


def _append(s):
    case, slots = s["case"], s["slots"]
    if own:
        from paper_2602_01901_b200 import quant

        quant.append(s["k_pool"], s["v_pool"], slots, s["k"], s["v"], case["page"])
        return quant.read(s["k_pool"], s["v_pool"], slots, case["kv_heads"], case["head_dim"], case["page"], s["k_back"], s["v_back"])
    heads, page, head_dim = case["kv_heads"], case["page"], case["head_dim"]
    n_codes = heads * page * head_dim // 2
    real = (slots >= 0)[:, None, None]
    spare = s["k_pool"].shape[0]                                        # a page of their own for slots that are none
    at = torch.where(slots >= 0, slots, spare * page).long()
    token, head = at[:, None] % page, torch.arange(heads, device=at.device)
    for which in "kv":
        pool, back = s[which + "_pool"], s[which + "_back"]
        codes, params = _quantise(s[which])
        # a byte's place inside a page, for every token, head and pair of elements
        inside = _places(which, head_dim, at.device)[at % page % 16]      # [tokens, 1, head_dim / 2]
        byte = (head[None] * page + token // 16 * 16)[..., None] * (head_dim // 2) + inside
        whole = torch.cat([pool, pool[:1]]).view(-1)
        base = (at // page * pool.shape[1])[:, None]
        whole[base[..., None] + byte] = codes[..., 0::2] | (codes[..., 1::2] << 4)
        word = (base + n_codes) // 4 + head[None] * page + token
        whole.view(torch.int32)[word] = params
        pool.copy_(whole.view(-1, pool.shape[1])[:-1])
        # and back
        held = pool.view(-1)[(base[..., None] + byte).clamp_(max=pool.numel() - 1)]
        words = pool.view(-1).view(torch.int32)[word.clamp_(max=pool.numel() // 4 - 1)]
        lo, r = (words << 16).view(torch.float32), (words & -65536).view(torch.float32)
        step = torch.where(r > 0, 1.0 / r, torch.zeros_like(r))
        values = lo[..., None] + torch.stack([held & 15, held >> 4], -1).flatten(-2).float() * step[..., None]
        back.copy_(torch.where(real, values.bfloat16(), back))
    return s["k_back"], s["v_back"]


def _places(which, head_dim, device):
    """[16 tokens, 1, head_dim / 2]: where in a block's bytes a pair of elements of a token lies."""
    shape, order = _AXES[which, head_dim]
    x = torch.arange(8 * head_dim, device=device).reshape(shape[:-1])
    return x.permute([i for i in order if i < len(shape) - 1]).reshape(16, 1, head_dim // 2)


def _attend(s):
    case = s["case"]
    if own:
        from paper_2602_01901_b200 import quant

        t, v = s["text"], s.get("visual")
        visual = quant.Stream(s["q_visual"], v["k_pool"], v["v_pool"], v["pages"], v["lens"]) if v else None
        return quant.attend(quant.Stream(s["q"], t["k_pool"], t["v_pool"], t["pages"], t["lens"]), case["kv_heads"], case["page"],
                            visual=visual, seq_ids=s["ids"], starts=s["starts"], max_queries=s["most"], causal=True)
    starts, rows = s["starts"].long(), s["ids"].long()
    n, heads, group, head_dim, most = case["seqs"], case["kv_heads"], case["group"], case["head_dim"], s["most"]
    count = starts[1:] - starts[:-1]
    place = torch.arange(most, device=starts.device)
    real = place < count[:, None]                                       # [sequence, query]
    at = (starts[:-1, None] + place).clamp_(max=s["q"].shape[0] - 1)
    scores, values, live = [], [], []
    for name, q in (("visual", s.get("q_visual")), ("text", s["q"])):
        if name not in s:
            continue
        t = s[name]
        ids = t["pages"][rows].clamp(min=0).long()
        length = t["lens"][rows].long()
        key = torch.arange(ids.shape[1] * case["page"], device=ids.device)
        seen = key < length[:, None]
        k = _values(t["k_pool"][ids], case, "k").flatten(1, 2)           # [sequence, token, head, d]
        v = _values(t["v_pool"][ids], case, "v").flatten(1, 2)
        k, v = (torch.where(seen[..., None, None], x, torch.zeros_like(x)) for x in (k, v))
        query = q[at].float().reshape(n, most, heads, group, head_dim).permute(0, 2, 1, 3, 4).reshape(n, heads, most * group, head_dim)
        dots = query @ k.permute(0, 2, 3, 1) / math.sqrt(head_dim)
        # the text stream ends with the queries' own tokens: a query sees what is not behind it
        last = length[:, None] - (count[:, None] - 1 - place if name == "text" else torch.zeros_like(place))
        visible = key < last[..., None]                                 # [sequence, query, token]
        scores.append(dots.reshape(n, heads, most, group, -1).masked_fill(~visible[:, None, :, None], -math.inf))
        values.append(v.permute(0, 2, 1, 3))
    score = torch.cat(scores, -1)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    total = weight.sum(-1, keepdim=True)
    out = weight.reshape(n, heads, most * group, -1) @ torch.cat(values, 2)
    out = out.reshape(n, heads, most, group, head_dim) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(total, -math.inf))[..., 0]
    out = out.permute(0, 2, 1, 3, 4).reshape(n, most, heads * group, head_dim)
    lse = lse.permute(0, 2, 1, 3).reshape(n, most, heads * group)
    # padded queries go to a row of their own behind the last
    to = torch.where(real, at, s["q"].shape[0])
    rows_out = torch.zeros(s["q"].shape[0] + 1, heads * group, head_dim, device=out.device)
    rows_lse = torch.zeros(s["q"].shape[0] + 1, heads * group, device=out.device)
    rows_out[to], rows_lse[to] = out, lse
    return rows_out[:-1].bfloat16(), rows_lse[:-1].contiguous()


def run(state):
    return {"tables": _tables, "append": _append, "attend": _attend}[state["case"]["op"]](state)


# ---- the definition in 64 bits, token by token's place ----------------------------------------------------------

def _held(pool, slots, case, which):
    """What the rows at ``slots`` stand for, fp64 [slots, heads, head_dim], each element looked up by its address."""
    heads, page, head_dim = case["kv_heads"], case["page"], case["head_dim"]
    flat = pool.reshape(-1)
    d = torch.arange(head_dim, device=flat.device)
    h = torch.arange(heads, device=flat.device)[:, None]
    tok = (slots % page)[:, None, None]
    i = tok % 16
    if which == "k":
        lane = (i // 2 * 4 + d // (head_dim // 4)) * 16
        inner = d // 2 % (head_dim // 8)
        byte = lane + inner + i % 2 * (512 if head_dim == 128 else 8)
    else:
        wide = d // (head_dim // 8)
        word = d // 2 % (head_dim // 16)
        byte = word // 4 * 512 + (wide * 4 + i // 4) * 16 + word % 4 * 4 + i % 4
    base = (slots // page)[:, None, None] * pool.shape[-1]
    codes = flat[base + (h * page + tok - i) * (head_dim // 2) + byte].long()
    codes = torch.where(d % 2 == 1, codes // 16, codes % 16).double()
    at = base[..., 0] + heads * page * (head_dim // 2) + (h[:, 0] * page + tok[..., 0]) * 4
    half = [flat[at + j].long() for j in range(4)]
    as_float = lambda a, b: ((a + 256 * b).to(torch.int32) << 16).view(torch.float32).double()
    lo, r = as_float(half[0], half[1]), as_float(half[2], half[3])
    return lo[..., None] + torch.where(r[..., None] > 0, codes / r[..., None], 0.0)


def exact(case, seed):
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    if case["op"] == "append":
        found = []
        for which in "kv":
            x = s[which].double()
            small, large = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            r = torch.where(large - small >= 2.0 ** -100, 15.0 / (large - small), 0.0).to(torch.bfloat16).double()
            steps = torch.round((x - small) * r)
            value = small + torch.where(r > 0, steps / torch.where(r > 0, r, 1.0), 0.0)
            found.append(torch.where((s["slots"] >= 0)[:, None, None], value, 0.0))
        return tuple(found)
    n, heads, group, head_dim, page = case["seqs"], case["kv_heads"], case["group"], case["head_dim"], case["page"]
    starts = s["starts"].tolist()
    out = torch.zeros(starts[-1], heads * group, head_dim, dtype=torch.float64, device=DEVICE)
    lse = torch.full((starts[-1], heads * group), -math.inf, dtype=torch.float64, device=DEVICE)
    for i in range(n):
        row, a, b = int(s["ids"][i]), starts[i], starts[i + 1]
        parts = [(s["text"], s["q"], True)] + ([(s["visual"], s["q_visual"], False)] if "visual" in s else [])
        for h0 in range(0, heads, 8):     # a few heads at a time: whole rows of a long sequence are large in 64 bits
            hs = list(range(h0, min(heads, h0 + 8)))
            logits, vals = [], []
            for t, q, is_text in parts:
                length = int(t["lens"][row])
                pos = torch.arange(length, device=DEVICE)
                slots = t["pages"][row].long()[pos // page] * page + pos % page
                key = torch.cat([_held(t["k_pool"], part, case, "k")[:, hs] for part in slots.split(4096)] or [torch.zeros(0, len(hs), head_dim, device=DEVICE, dtype=torch.float64)])
                val = torch.cat([_held(t["v_pool"], part, case, "v")[:, hs] for part in slots.split(4096)] or [torch.zeros(0, len(hs), head_dim, device=DEVICE, dtype=torch.float64)])
                qs = q[a:b].double().reshape(b - a, heads, group, head_dim)[:, hs]
                dot = torch.einsum("nhgd,lhd->nhgl", qs, key) / math.sqrt(head_dim)
                if is_text:
                    behind = pos[None] > (length - (b - a) + torch.arange(b - a, device=DEVICE))[:, None]
                    dot = torch.where(behind[:, None, None], -math.inf, dot)
                logits.append(dot)
                vals.append(val)
            logit, val = torch.cat(logits, -1), torch.cat(vals, 0)
            if logit.shape[-1] == 0:
                continue
            total = torch.logsumexp(logit, -1)
            weight = torch.where(total[..., None].isfinite(), torch.exp(logit - total[..., None]), 0.0)
            cols = slice(hs[0] * group, (hs[-1] + 1) * group)
            out[a:b, cols] = torch.einsum("nhgl,lhd->nhgd", weight, val).reshape(b - a, -1, head_dim)
            lse[a:b, cols] = total.reshape(b - a, -1)
    return out, lse
