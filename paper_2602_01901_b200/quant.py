"""A K/V cache in 4 bits: page tables that grow on the device, rows quantised into pages, attention over them.

The calls of ``include/qc.h`` on torch tensors: every buffer is the caller's, every call is enqueued on the current
stream of the tensors' device and returns at once, and nothing is kept between calls, so a step can be captured into a
``torch.cuda.graph`` and replayed while its sequences grow.  Arguments that a call can see on the host are checked here
or by the library (``ValueError``, ``QcError``); numbers on the device (ids, lengths, pages) are checked there and end in
the table's status word (``PageTable.check``).

    table = PageTable.empty(max_seqs, max_pages, page_size, n_pages)
    k_pool, v_pool = (empty_pool(n_kv_heads, head_dim, page_size, n_pages) for _ in "kv")      # of each layer
    starts, slots = table_extend(table, n_new, seq_ids=ids, max_slots=n_tokens)                # once a step
    append(k_pool, v_pool, slots, k, v, page_size)                                             # each layer
    out, lse = attend(Stream(q, k_pool, v_pool, table.pages, table.lens), n_kv_heads, page_size,
                      seq_ids=ids, starts=starts, max_queries=most)
    table_trim(table, lengths, seq_ids=ids)                                                    # drafts turned down
"""

from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from . import binding as qc


def _stream_of(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _ints(t: Optional[torch.Tensor], name: str, device: torch.device, count: Optional[int] = None) -> int:
    """Device address of a dense int32 tensor (0 for None)."""
    if t is None:
        return 0
    if t.dtype is not torch.int32 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} has to be a dense int32 tensor on {device}")
    if count is not None and t.numel() != count:
        raise ValueError(f"{name} has {t.numel()} entries, not {count}")
    return t.data_ptr()


def _on_gpu(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} has to be on a CUDA device (there is no CPU fallback)")
    return t.device


class PageTable:
    """Page table of one stream (``qc_table``) over the caller's int32 tensors: ``pages`` [max_seqs, max_pages],
    ``lens`` [max_seqs], ``free`` [n_pages], ``state`` [4]."""

    __slots__ = ("pages", "lens", "free", "state", "page_size", "device", "c")

    def __init__(self, pages: torch.Tensor, lens: torch.Tensor, free: torch.Tensor, state: torch.Tensor, page_size: int):
        device = _on_gpu(pages, "pages")
        if pages.dim() != 2:
            raise ValueError("pages has to be [max_seqs, max_pages]")
        max_seqs, max_pages = pages.shape
        self.pages, self.lens, self.free, self.state, self.page_size, self.device = pages, lens, free, state, page_size, device
        self.c = qc.qc_table(max_seqs, max_pages, page_size, free.numel(), _ints(pages, "pages", device), _ints(lens, "lens", device, max_seqs),
                             _ints(free, "free", device), _ints(state, "state", device, 4))

    @classmethod
    def empty(cls, max_seqs: int, max_pages: int, page_size: int, n_pages: int, device=0) -> "PageTable":
        make = lambda *shape: torch.empty(shape, dtype=torch.int32, device=torch.device("cuda", device) if isinstance(device, int) else device)
        table = cls(make(max_seqs, max_pages), make(max_seqs), make(n_pages), make(4), page_size)
        table.reset()
        return table

    def reset(self) -> None:
        qc.qc_table_reset(self.device.index, _stream_of(self.pages), self.c)

    def check(self) -> None:
        """Raises what the status word holds (waits for the stream)."""
        status = int(self.state[1])
        if status != qc.QC_OK:
            raise qc.QcError(status, "page table")


def _batch(table: PageTable, seq_ids, counts, name: str, n_seqs):
    listed = seq_ids if seq_ids is not None else counts
    n = listed.numel() if listed is not None else table.c.max_seqs if n_seqs is None else n_seqs
    if n_seqs is not None and n_seqs != n:
        raise ValueError(f"n_seqs is {n_seqs}, but {n} sequences are listed")
    return n, _ints(seq_ids, "seq_ids", table.device, n), _ints(counts, name, table.device, n)


def table_extend(table: PageTable, n_new: Optional[torch.Tensor] = None, *, seq_ids: Optional[torch.Tensor] = None,
                 n_seqs: Optional[int] = None, max_slots: Optional[int] = None):
    """``n_new[i]`` (None: 1) more tokens for row ``seq_ids[i]`` (None: i).  Returns (starts [n + 1], slots [max_slots]):
    sequence i's new tokens are ``starts[i]`` to ``starts[i + 1] - 1`` of the call, token t goes to ``slots[t]``, and slots
    behind the last token are -1.  ``max_slots`` may be left out where every sequence takes one token."""
    n, ids, new = _batch(table, seq_ids, n_new, "n_new", n_seqs)
    if max_slots is None:
        if n_new is not None:
            raise ValueError("max_slots: the most tokens that the call may add")
        max_slots = n
    starts = torch.empty(n + 1, dtype=torch.int32, device=table.device)
    slots = torch.empty(max_slots, dtype=torch.int32, device=table.device)
    qc.qc_table_extend(table.device.index, _stream_of(starts), table.c, n, ids, new, max_slots, starts.data_ptr(), slots.data_ptr())
    return starts, slots


def table_trim(table: PageTable, n_keep: Optional[torch.Tensor] = None, *, seq_ids: Optional[torch.Tensor] = None,
               n_seqs: Optional[int] = None) -> None:
    """Row ``seq_ids[i]`` (None: i) keeps its first ``n_keep[i]`` tokens (None: none, the sequence is released)."""
    n, ids, keep = _batch(table, seq_ids, n_keep, "n_keep", n_seqs)
    qc.qc_table_trim(table.device.index, _stream_of(table.pages), table.c, n, ids, keep)


def page_bytes(n_kv_heads: int, head_dim: int, page_size: int) -> int:
    return qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, 1))


def empty_pool(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, device=0) -> torch.Tensor:
    """A pool for one tensor (K or V) of one layer and stream: uint8 [n_pages, page bytes], not initialised."""
    size = qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, n_pages))
    return torch.empty((n_pages, size // n_pages), dtype=torch.uint8, device=torch.device("cuda", device) if isinstance(device, int) else device)


def _pool(t: torch.Tensor, name: str, heads: int, head_dim: int, page_size: int, device: torch.device) -> int:
    if t.dtype is not torch.uint8 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} has to be a dense uint8 tensor on {device}")
    if t.dim() != 2 or t.shape[1] != heads * page_size * (head_dim // 2 + 4):
        raise ValueError(f"{name} has to be [pages, {heads * page_size * (head_dim // 2 + 4)}] for {heads} heads of {head_dim} and pages of {page_size}")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, device: torch.device) -> tuple:
    """(address, token stride) of bf16 [tokens, heads, head_dim] rows whose heads are dense (0 for a single token)."""
    if t.dtype is not torch.bfloat16 or t.dim() != 3 or t.device != device:
        raise ValueError(f"{name} has to be a bfloat16 tensor [tokens, heads, head_dim] on {device}")
    stride = t.stride()
    if (stride[2] != 1 and t.shape[2] > 1) or (stride[1] != t.shape[2] and t.shape[1] > 1):
        raise ValueError(f"{name}: the heads of a token have to be dense")
    return t.data_ptr(), stride[0] if t.shape[0] > 1 else 0


def append(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, k: Optional[torch.Tensor],
           v: Optional[torch.Tensor], page_size: int) -> None:
    """Quantises rows ``k``, ``v`` (bf16 [tokens, heads, head_dim]; heads dense, tokens any stride that is a multiple of 8)
    into the pools at ``slots``; negative slots are left out.  Either pair may be None (a lazy layer that stores no K)."""
    rows = k if k is not None else v
    if rows is None or (k is None) != (k_pool is None) or (v is None) != (v_pool is None):
        raise ValueError("a pool for every tensor, and one of k and v at least")
    device = _on_gpu(rows, "k" if k is not None else "v")
    tokens, heads, head_dim = rows.shape if rows.dim() == 3 else (0, 0, 0)
    k_at = v_at = kp = vp = k_stride = v_stride = 0
    pool = k_pool if k is not None else v_pool
    if k is not None:
        k_at, k_stride = _rows(k, "k", device)
        kp = _pool(k_pool, "k_pool", heads, head_dim, page_size, device)
    if v is not None:
        v_at, v_stride = _rows(v, "v", device)
        vp = _pool(v_pool, "v_pool", heads, head_dim, page_size, device)
        if k is not None and (k.shape != v.shape or k_pool.shape != v_pool.shape):
            raise ValueError("k and v, and their pools, have to have the same shape")
    if tokens == 0:
        return
    qc.qc_quant_append(device.index, _stream_of(rows), qc.qc_quant_shape(heads, head_dim, page_size, pool.shape[0]), tokens,
                       _ints(slots, "slots", device, tokens), k_at, k_stride, v_at, v_stride, kp, vp)


def read(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, n_kv_heads: int, head_dim: int,
         page_size: int, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """What the rows at ``slots`` stand for: (k, v), bf16 [tokens, n_kv_heads, head_dim], None for a pool that is None.
    Rows of negative slots stay what they were in ``k_out`` / ``v_out`` (zeros where those are made here)."""
    device = _on_gpu(slots, "slots")
    tokens, at = slots.numel(), _ints(slots, "slots", device)
    if k_pool is None and v_pool is None:
        raise ValueError("one of k_pool and v_pool at least")
    outs, ptrs, pools = [], [], []
    for pool, out, name in ((k_pool, k_out, "k"), (v_pool, v_out, "v")):
        if pool is None:
            outs.append(None), ptrs.append(0), pools.append(0)
            continue
        pools.append(_pool(pool, name + "_pool", n_kv_heads, head_dim, page_size, device))
        if out is None:
            out = torch.zeros((tokens, n_kv_heads, head_dim), dtype=torch.bfloat16, device=device)
        elif out.shape != (tokens, n_kv_heads, head_dim) or out.dtype is not torch.bfloat16 or not out.is_contiguous() or out.device != device:
            raise ValueError(f"{name}_out has to be a dense bfloat16 tensor {(tokens, n_kv_heads, head_dim)} on {device}")
        outs.append(out), ptrs.append(out.data_ptr())
    if k_pool is not None and v_pool is not None and k_pool.shape != v_pool.shape:
        raise ValueError("the pools have to have the same shape")
    if tokens:
        shape = qc.qc_quant_shape(n_kv_heads, head_dim, page_size, (k_pool if k_pool is not None else v_pool).shape[0])
        qc.qc_quant_read(device.index, _stream_of(slots), shape, tokens, at, pools[0], pools[1], ptrs[0], ptrs[1])
    return outs[0], outs[1]


class Stream(NamedTuple):
    """One stream of a cache as ``attend`` reads it: the queries that score its keys (bf16 [tokens, query heads, head_dim]),
    its pools, its table's pages and lengths."""

    q: torch.Tensor
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    pages: torch.Tensor
    lens: torch.Tensor


def _stream(s: Stream, name: str, heads: int, page_size: int, shape, rows: Optional[int], device: torch.device):
    at, stride = _rows(s.q, name + ".q", device)
    if s.q.shape != shape:
        raise ValueError(f"{name}.q has to be {tuple(shape)}")
    if s.pages.dim() != 2 or (rows is not None and s.pages.shape[0] != rows) or s.k_pool.shape != s.v_pool.shape:
        raise ValueError(f"{name}: pages has to be [sequences, pages] with as many rows as the other stream's, the pools of one shape")
    return qc.qc_quant_stream(at, stride, _pool(s.k_pool, name + ".k_pool", heads, shape[2], page_size, device),
                              _pool(s.v_pool, name + ".v_pool", heads, shape[2], page_size, device), _ints(s.pages, name + ".pages", device),
                              _ints(s.lens, name + ".lens", device, s.pages.shape[0]), s.pages.shape[1], s.k_pool.shape[0])


def attend(text: Stream, n_kv_heads: int, page_size: int, *, visual: Optional[Stream] = None, seq_ids: Optional[torch.Tensor] = None,
           starts: Optional[torch.Tensor] = None, max_queries: int = 1, causal: bool = True, scale: float = 0.0,
           out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Attention of each sequence's query tokens over its cached rows, the queries' own among them (``qc_quant_attend``):
    one softmax over the visual stream's keys, scored by ``visual.q``, and the text stream's, scored by ``text.q``.
    Sequence i is row ``seq_ids[i]`` (None: i) of the tables and has query tokens ``starts[i]`` to ``starts[i + 1] - 1`` (None:
    token i), ``max_queries`` at most.  ``causal``: they are the last tokens of the text stream, and none sees what is behind
    it.  Returns (out bf16 [tokens, query heads, head_dim], lse fp32 [tokens, query heads]); a query that sees nothing gets 0
    and minus infinity.  ``status``: an int32 word for what is met on the device (a ``PageTable``'s ``state[1:2]``)."""
    q = text.q
    device = _on_gpu(q, "text.q")
    if q.dim() != 3:
        raise ValueError("text.q has to be [tokens, heads, head_dim]")
    shape = q.shape
    tokens, q_heads, head_dim = shape
    t = _stream(text, "text", n_kv_heads, page_size, shape, None, device)
    rows = text.pages.shape[0]
    v = _stream(visual, "visual", n_kv_heads, page_size, shape, rows, device) if visual is not None else None
    n = seq_ids.numel() if seq_ids is not None else starts.numel() - 1 if starts is not None else tokens
    if out is None:
        out = torch.empty(shape, dtype=torch.bfloat16, device=device)
    elif out.shape != shape or out.dtype is not torch.bfloat16 or not out.is_contiguous() or out.device != device:
        raise ValueError(f"out has to be a dense bfloat16 tensor {tuple(shape)} on {device}")
    lse = torch.empty((tokens, q_heads), dtype=torch.float32, device=device)
    args = qc.qc_quant_attend_args(q_heads, n_kv_heads, head_dim, page_size, n, rows, tokens, max_queries, bool(causal), scale,
                                   _ints(seq_ids, "seq_ids", device, n), _ints(starts, "starts", device, n + 1), C.pointer(t),
                                   C.pointer(v) if v is not None else None, out.data_ptr(), lse.data_ptr(), 0, 0,
                                   _ints(status, "status", device, 1))
    need = qc.qc_quant_workspace_bytes(args)
    if need:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        args.workspace_dev, args.workspace_bytes = workspace.data_ptr(), need
    if tokens:
        qc.qc_quant_attend(device.index, _stream_of(q), args)
    return out, lse
