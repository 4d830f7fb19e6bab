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

import struct
from typing import NamedTuple, Optional

import torch

from . import binding as qc

# The structures of include/qc.h, packed (native sizes and alignment).
_TABLE = struct.Struct("@4i4P")
_SHAPE = struct.Struct("@4i")
_STREAM = "Pq4P2i"
_ATTEND = struct.Struct("@9if2P" + 2 * _STREAM + "3PNP")
_NO_STREAM = (0,) * 8

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_int32, _uint8, _bf16 = torch.int32, torch.uint8, torch.bfloat16
_lib = None


def _library():
    global _lib
    if _lib is None:
        _lib = qc.load()
    return _lib


def _check(status: int, where: str) -> None:
    if status:
        raise qc.QcError(status, where)


def _device_of(t: torch.Tensor, name: str) -> int:
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} has to be on a CUDA device (there is no CPU fallback)")
    return index


def _ints(t: Optional[torch.Tensor], name: str, index: int, count: Optional[int] = None) -> int:
    """Device address of a dense int32 tensor (0 for None)."""
    if t is None:
        return 0
    if t.dtype is not _int32 or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} has to be a dense int32 tensor on cuda:{index}")
    if count is not None and t.numel() != count:
        raise ValueError(f"{name} has {t.numel()} entries, not {count}")
    return t.data_ptr()


class PageTable:
    """Page table of one stream (``qc_table``) over the caller's int32 tensors: ``pages`` [max_seqs, max_pages],
    ``lens`` [max_seqs], ``free`` [n_pages], ``state`` [4]."""

    __slots__ = ("pages", "lens", "free", "state", "page_size", "index", "max_seqs", "packed")

    def __init__(self, pages: torch.Tensor, lens: torch.Tensor, free: torch.Tensor, state: torch.Tensor, page_size: int):
        index = _device_of(pages, "pages")
        if pages.dim() != 2:
            raise ValueError("pages has to be [max_seqs, max_pages]")
        max_seqs, max_pages = pages.shape
        self.pages, self.lens, self.free, self.state, self.page_size, self.index, self.max_seqs = pages, lens, free, state, page_size, index, max_seqs
        self.packed = _TABLE.pack(max_seqs, max_pages, page_size, free.numel(), _ints(pages, "pages", index), _ints(lens, "lens", index, max_seqs),
                                  _ints(free, "free", index), _ints(state, "state", index, 4))

    @classmethod
    def empty(cls, max_seqs: int, max_pages: int, page_size: int, n_pages: int, device=0) -> "PageTable":
        make = lambda *shape: torch.empty(shape, dtype=_int32, device=torch.device("cuda", device) if isinstance(device, int) else device)
        table = cls(make(max_seqs, max_pages), make(max_seqs), make(n_pages), make(4), page_size)
        table.reset()
        return table

    def reset(self) -> None:
        _check(_library().qc_table_reset(self.index, _raw_stream(self.index), self.packed), "qc_table_reset")

    def check(self) -> None:
        """Raises what the status word holds (waits for the stream)."""
        _check(int(self.state[1]), "page table")


def _batch(table: PageTable, seq_ids, counts, name: str, n_seqs):
    listed = seq_ids if seq_ids is not None else counts
    n = listed.numel() if listed is not None else table.max_seqs if n_seqs is None else n_seqs
    if n_seqs is not None and n_seqs != n:
        raise ValueError(f"n_seqs is {n_seqs}, but {n} sequences are listed")
    return n, _ints(seq_ids, "seq_ids", table.index, n), _ints(counts, name, table.index, n)


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
    starts, slots = table.lens.new_empty(n + 1), table.lens.new_empty(max_slots)
    index = table.index
    _check(_library().qc_table_extend(index, _raw_stream(index), table.packed, n, ids, new, max_slots, starts.data_ptr(), slots.data_ptr()),
           "qc_table_extend")
    return starts, slots


def table_trim(table: PageTable, n_keep: Optional[torch.Tensor] = None, *, seq_ids: Optional[torch.Tensor] = None,
               n_seqs: Optional[int] = None) -> None:
    """Row ``seq_ids[i]`` (None: i) keeps its first ``n_keep[i]`` tokens (None: none, the sequence is released)."""
    n, ids, keep = _batch(table, seq_ids, n_keep, "n_keep", n_seqs)
    index = table.index
    _check(_library().qc_table_trim(index, _raw_stream(index), table.packed, n, ids, keep), "qc_table_trim")


def page_bytes(n_kv_heads: int, head_dim: int, page_size: int) -> int:
    return qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, 1))


def empty_pool(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, device=0) -> torch.Tensor:
    """A pool for one tensor (K or V) of one layer and stream: uint8 [n_pages, page bytes], not initialised."""
    size = qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, n_pages))
    return torch.empty((n_pages, size // n_pages), dtype=_uint8, device=torch.device("cuda", device) if isinstance(device, int) else device)


def _pool(t: torch.Tensor, name: str, row: int, index: int) -> int:
    """Device address of a pool whose pages have ``row`` bytes."""
    if t.dtype is not _uint8 or t.get_device() != index or not t.is_contiguous() or t.dim() != 2 or t.shape[1] != row:
        raise ValueError(f"{name} has to be a dense uint8 tensor [pages, {row}] on cuda:{index} (heads * page size * (head_dim / 2 + 4) bytes a page)")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, index: int) -> int:
    """Token stride of bf16 [tokens, heads, head_dim] rows whose heads are dense (0 for a single token)."""
    if t.dtype is not _bf16 or t.dim() != 3 or t.get_device() != index:
        raise ValueError(f"{name} has to be a bfloat16 tensor [tokens, heads, head_dim] on cuda:{index}")
    tokens, heads, width = t.shape
    stride, head, one = t.stride()
    if (one != 1 and width > 1) or (head != width and heads > 1):
        raise ValueError(f"{name}: the heads of a token have to be dense")
    return stride if tokens > 1 else 0


def append(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, k: Optional[torch.Tensor],
           v: Optional[torch.Tensor], page_size: int) -> None:
    """Quantises rows ``k``, ``v`` (bf16 [tokens, heads, head_dim]; heads dense, tokens any stride that is a multiple of 8)
    into the pools at ``slots``; negative slots are left out.  Either pair may be None (a lazy layer that stores no K)."""
    rows, pool = (k, k_pool) if k is not None else (v, v_pool)
    if rows is None or (k is None) != (k_pool is None) or (v is None) != (v_pool is None):
        raise ValueError("a pool for every tensor, and one of k and v at least")
    index = _device_of(rows, "k" if k is not None else "v")
    if rows.dim() != 3:
        raise ValueError("k and v have to be [tokens, heads, head_dim]")
    tokens, heads, head_dim = rows.shape
    row = heads * page_size * (head_dim // 2 + 4)
    k_at = v_at = kp = vp = k_stride = v_stride = 0
    if k is not None:
        k_at, k_stride, kp = k.data_ptr(), _rows(k, "k", index), _pool(k_pool, "k_pool", row, index)
    if v is not None:
        v_at, v_stride, vp = v.data_ptr(), _rows(v, "v", index), _pool(v_pool, "v_pool", row, index)
        if k is not None and (k.shape != v.shape or k_pool.shape != v_pool.shape):
            raise ValueError("k and v, and their pools, have to have the same shape")
    at = _ints(slots, "slots", index, tokens)
    if tokens:
        _check(_library().qc_quant_append(index, _raw_stream(index), _SHAPE.pack(heads, head_dim, page_size, pool.shape[0]), tokens, at, k_at, k_stride,
                                          v_at, v_stride, kp, vp), "qc_quant_append")


def _out(out: Optional[torch.Tensor], shape: tuple, like: torch.Tensor, name: str, index: int) -> torch.Tensor:
    if out is None:
        return torch.zeros(shape, dtype=_bf16, device=like.device)
    if out.shape != shape or out.dtype is not _bf16 or out.get_device() != index or not out.is_contiguous():
        raise ValueError(f"{name} has to be a dense bfloat16 tensor {shape} on cuda:{index}")
    return out


def read(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, n_kv_heads: int, head_dim: int,
         page_size: int, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """What the rows at ``slots`` stand for: (k, v), bf16 [tokens, n_kv_heads, head_dim], None for a pool that is None.
    Rows of negative slots stay what they were in ``k_out`` / ``v_out`` (zeros where those are made here)."""
    index = _device_of(slots, "slots")
    tokens, at = slots.numel(), _ints(slots, "slots", index)
    pool = k_pool if k_pool is not None else v_pool
    if pool is None:
        raise ValueError("one of k_pool and v_pool at least")
    row, shape = n_kv_heads * page_size * (head_dim // 2 + 4), (tokens, n_kv_heads, head_dim)
    k_at = v_at = kp = vp = 0
    if k_pool is None:
        k_out = None
    else:
        kp, k_out = _pool(k_pool, "k_pool", row, index), _out(k_out, shape, slots, "k_out", index)
        k_at = k_out.data_ptr()
    if v_pool is None:
        v_out = None
    else:
        vp, v_out = _pool(v_pool, "v_pool", row, index), _out(v_out, shape, slots, "v_out", index)
        v_at = v_out.data_ptr()
        if v_pool.shape != pool.shape:
            raise ValueError("the pools have to have the same shape")
    if tokens:
        _check(_library().qc_quant_read(index, _raw_stream(index), _SHAPE.pack(n_kv_heads, head_dim, page_size, pool.shape[0]), tokens, at, kp, vp, k_at,
                                        v_at), "qc_quant_read")
    return k_out, v_out


class Stream(NamedTuple):
    """One stream of a cache as ``attend`` reads it: the queries that score its keys (bf16 [tokens, query heads, head_dim]),
    its pools, its table's pages and lengths."""

    q: torch.Tensor
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    pages: torch.Tensor
    lens: torch.Tensor


def _stream(s: Stream, name: str, row: int, shape, rows: Optional[int], index: int) -> tuple:
    q, k_pool, v_pool, pages, lens = s
    stride = _rows(q, name + ".q", index)
    if q.shape != shape:
        raise ValueError(f"{name}.q has to be {tuple(shape)}")
    if pages.dim() != 2 or (rows is not None and pages.shape[0] != rows):
        raise ValueError(f"{name}.pages has to be [sequences, pages], with as many rows as the other stream's")
    kp, vp = _pool(k_pool, name + ".k_pool", row, index), _pool(v_pool, name + ".v_pool", row, index)
    n_pages = k_pool.shape[0]
    if v_pool.shape[0] != n_pages:
        raise ValueError(f"{name}: the pools have to have the same shape")
    n, width = pages.shape
    return q.data_ptr(), stride, kp, vp, _ints(pages, name + ".pages", index), _ints(lens, name + ".lens", index, n), width, n_pages


_workspaces: dict = {}     # bytes by (head_dim, rows of queries per KV head are more than 8)


def _workspace_bytes(head_dim: int, q_heads: int, n_kv_heads: int, page_size: int, max_queries: int) -> int:
    key = (head_dim, q_heads, n_kv_heads, page_size, max_queries)
    size = _workspaces.get(key)
    if size is None:
        args = qc.qc_quant_attend_args(n_q_heads=q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, page_size=page_size, n_seqs=1, max_seqs=1,
                                       max_queries=max_queries)
        size = _workspaces[key] = qc.qc_quant_workspace_bytes(args)
    return size


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
    index = _device_of(q, "text.q")
    if q.dim() != 3:
        raise ValueError("text.q has to be [tokens, heads, head_dim]")
    shape = q.shape
    tokens, q_heads, head_dim = shape
    row = n_kv_heads * page_size * (head_dim // 2 + 4)
    t = _stream(text, "text", row, shape, None, index)
    rows = text.pages.shape[0]
    v = _NO_STREAM if visual is None else _stream(visual, "visual", row, shape, rows, index)
    n = seq_ids.numel() if seq_ids is not None else starts.numel() - 1 if starts is not None else tokens
    if out is None:
        out = q.new_empty(shape)
    elif out.shape != shape or out.dtype is not _bf16 or out.get_device() != index or not out.is_contiguous():
        raise ValueError(f"out has to be a dense bfloat16 tensor {tuple(shape)} on cuda:{index}")
    lse = torch.empty((tokens, q_heads), dtype=torch.float32, device=q.device)
    size = _workspace_bytes(head_dim, q_heads, n_kv_heads, page_size, max_queries)
    workspace = torch.empty(size, dtype=_uint8, device=q.device)
    ids, begin, word = _ints(seq_ids, "seq_ids", index, n), _ints(starts, "starts", index, n + 1), _ints(status, "status", index, 1)
    if tokens:
        packed = _ATTEND.pack(q_heads, n_kv_heads, head_dim, page_size, n, rows, tokens, max_queries, bool(causal), scale, ids, begin, *t, *v, out.data_ptr(),
                              lse.data_ptr(), workspace.data_ptr(), size, word)
        _check(_library().qc_quant_attend(index, _raw_stream(index), packed), "qc_quant_attend")
    return out, lse
