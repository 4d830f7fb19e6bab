"""Replays of a captured attention call: a replay whose lengths were changed while it ran may be wrong itself, the next one is
right again; and what the workspace holds before a replay does not matter."""

import pytest
import torch

from paper_2602_01901_b200 import binding as qc
from paper_2602_01901_b200 import quant

from quant_util import DEV, gen
from test_gpu_quant_attend import i32

pytestmark = pytest.mark.gpu


def cache(lens, kv_heads, group, head_dim, page, seed):
    g, per = gen(seed), -(-max(lens) // page) + 1
    table = quant.PageTable.empty(len(lens), per, page, len(lens) * per)
    pools = [quant.empty_pool(kv_heads, head_dim, page, len(lens) * per) for _ in "kv"]
    _, slots = quant.table_extend(table, i32(lens), max_slots=sum(lens))
    k, v = (torch.randn(sum(lens), kv_heads, head_dim, generator=g).bfloat16().to(DEV) for _ in "kv")
    quant.append(*pools, slots, k, v, page)
    q = torch.randn(len(lens), kv_heads * group, head_dim, generator=g).bfloat16().to(DEV)
    return quant.Stream(q, *pools, table.pages, table.lens)


# units in the ranges of several teams, of single warps and of whole blocks, of 2, 4 and 8 and of 16 rows
SHAPES = [([9001, 5000, 7333], 2, 4, 64), ([30000], 1, 1, 128), ([1900] * 30, 8, 1, 128), ([6000, 9000], 2, 16, 128), ([3000, 100, 2500, 4000] * 4, 4, 8, 64)]


@pytest.mark.parametrize("lens,kv_heads,group,head_dim", SHAPES, ids=[f"{len(s[0])}x{s[1]}x{s[2]}" for s in SHAPES])
def test_lengths_that_change_under_a_replay_cost_that_replay_alone(lens, kv_heads, group, head_dim):
    """(Rows of K and V are there for every length that is set; other lengths are other plans of who takes which part.)"""
    stream = cache(lens, kv_heads, group, head_dim, 32, 5)
    right = stream.lens.clone()
    want, want_lse = quant.attend(stream, kv_heads, 32)
    graph, changes = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = quant.attend(stream, kv_heads, 32)      # (one call, whose workspace no other one writes)
    with torch.cuda.graph(changes):
        for by in (2, 3, 5, 2, 7, 3, 2, 9) * 30:
            torch.div(right, by, rounding_mode="floor", out=stream.lens)
            torch.mul(right, 1, out=stream.lens)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(150):
        for side, work, times in zip(sides, (graph, changes), (30, 1)):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for _ in range(times):
                    work.replay()
        torch.cuda.synchronize()
        assert torch.equal(stream.lens, right)
        for _ in range(2):      # the lengths stay what they are
            out.fill_(7)
            graph.replay()
            assert torch.equal(out, want) and torch.equal(lse, want_lse), turn


@pytest.mark.parametrize("lens,kv_heads,group,head_dim", SHAPES, ids=[f"{len(s[0])}x{s[1]}x{s[2]}" for s in SHAPES])
def test_a_replay_does_not_look_at_what_its_workspace_held(lens, kv_heads, group, head_dim):
    stream = cache(lens, kv_heads, group, head_dim, 32, 6)
    q = stream.q
    want, want_lse = quant.attend(stream, kv_heads, 32)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    part = qc.qc_quant_stream(q_dev=q.data_ptr(), q_stride=q.stride(0), k_pool_dev=stream.k_pool.data_ptr(), v_pool_dev=stream.v_pool.data_ptr(),
                              pages_dev=stream.pages.data_ptr(), lens_dev=stream.lens.data_ptr(), max_pages=stream.pages.shape[1], n_pages=stream.k_pool.shape[0])
    args = qc.qc_quant_attend_args(n_q_heads=q.shape[1], n_kv_heads=kv_heads, head_dim=head_dim, page_size=32, n_seqs=len(lens), max_seqs=len(lens),
                                   n_tokens=len(lens), max_queries=1, causal=1, text=part, out_dev=out.data_ptr(), lse_out_dev=lse.data_ptr())
    args.workspace_bytes = qc.qc_quant_workspace_bytes(args)
    workspace = torch.zeros(args.workspace_bytes, dtype=torch.uint8, device=DEV)
    args.workspace_dev = workspace.data_ptr()
    qc.qc_quant_attend(0, torch.cuda.current_stream().cuda_stream, args)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]      # which share the workspace, one replay at a time
    for graph in graphs:
        with torch.cuda.graph(graph):
            qc.qc_quant_attend(0, torch.cuda.current_stream().cuda_stream, args)
    g = torch.Generator(DEV)
    g.manual_seed(1)
    fills = [lambda: workspace.zero_(), lambda: workspace.fill_(0xFF), lambda: workspace.random_(0, 256, generator=g), lambda: workspace[:4096].random_(0, 256, generator=g),
             lambda: workspace[::7].zero_(), lambda: None, lambda: workspace.view(torch.int32).copy_(torch.arange(workspace.numel() // 4, device=DEV, dtype=torch.int32))]
    for turn in range(70):
        fills[turn % len(fills)]()
        for _ in range(1 + turn % 3):
            out.fill_(7), lse.fill_(7)
            graphs[turn // 2 % 2].replay()
            assert torch.equal(out, want) and torch.equal(lse, want_lse), turn


def test_thousands_of_replays_in_a_workspace_of_their_own():
    stream = cache([9001, 5000, 7333], 2, 4, 64, 32, 5)
    want, want_lse = quant.attend(stream, 2, 32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = quant.attend(stream, 2, 32)
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(8000):      # more than a workspace counts before it begins again, twice
        graph.replay()
        wrong += (out != want).sum() + (lse != want_lse).sum()
        out.fill_(7)
    assert int(wrong) == 0


@pytest.mark.parametrize("lens,kv_heads,group,head_dim", SHAPES, ids=[f"{len(s[0])}x{s[1]}x{s[2]}" for s in SHAPES])
def test_lengths_that_change_between_replays(lens, kv_heads, group, head_dim):
    """Plans of every kind after one another in one workspace: the bits of a call that is not captured."""
    stream = cache(lens, kv_heads, group, head_dim, 32, 7)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = quant.attend(stream, kv_heads, 32)
    g = gen(9)
    for turn in range(60):
        top = [1.0, 0.02, 0.3][turn % 3]
        now = (torch.tensor(lens) * top * torch.rand(len(lens), generator=g)).to(torch.int32)
        stream.lens.copy_(now.to(DEV))
        want, want_lse = quant.attend(stream, kv_heads, 32)
        out.fill_(7), lse.fill_(7)
        graph.replay()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), turn
