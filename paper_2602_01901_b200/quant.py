"""A K/V cache in 4 bits: page tables that grow on the device, rows quantised into pages, attention over them.

The calls of ``include/qc.h`` on torch tensors: every buffer is the caller's, every call is enqueued on the current
stream of the tensors' device and returns at once, and nothing is kept between calls, so a step can be captured into a
``torch.cuda.graph`` and replayed while its sequences grow.  Arguments that a call can see on the host are checked here
or by the library (``ValueError``, ``QcError``); numbers on the device (ids, lengths, pages) are checked there and end in
the table's status word (``PageTable.check``).  No gradient flows through any of them.

    table = PageTable.empty(max_seqs, max_pages, page_size, n_pages)
    k_pool, v_pool = (empty_pool(n_kv_heads, head_dim, page_size, n_pages) for _ in "kv")      # of each layer
    starts, slots = table_extend(table, n_new, seq_ids=ids, max_slots=n_tokens)                # once a step
    append(k_pool, v_pool, slots, k, v, page_size)                                             # each layer
    out, lse = attend(Stream(q, k_pool, v_pool, table.pages, table.lens), n_kv_heads, page_size,
                      seq_ids=ids, starts=starts, max_queries=most)
    table_trim(table, lengths, seq_ids=ids)                                                    # drafts turned down
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as qc
from .build import built_for

_calls = None


def _native():
    """The compiled calls (csrc/qc_torch.cpp); raises if they have not been built."""
    global _calls
    if _calls is None:
        qc.load()
        try:
            from . import _qc_torch
        except ImportError as e:
            raise RuntimeError(f"{e}: build it with `python -m paper_2602_01901_b200.build` (there is no CPU or PyTorch fallback)") from e
        made_for = getattr(_qc_torch, "built_for", "_qc_torch of an earlier build;")
        if made_for != f"_qc_torch for {built_for()};":
            raise RuntimeError(f"{made_for} this is {built_for()}: build it again with `python -m paper_2602_01901_b200.build`")
        _qc_torch.error_class(qc.QcError)
        _calls = _qc_torch
    return _calls


def _cuda(device) -> torch.device:
    return torch.device("cuda", device) if isinstance(device, int) else torch.device(device)


class PageTable:
    """Page table of one stream (``qc_table``) over the caller's int32 tensors: ``pages`` [max_seqs, max_pages],
    ``lens`` [max_seqs], ``free`` [n_pages], ``state`` [4].  It is these tensors for good: others make another table."""

    __slots__ = ("pages", "lens", "free", "state", "page_size", "packed")

    def __init__(self, pages: torch.Tensor, lens: torch.Tensor, free: torch.Tensor, state: torch.Tensor, page_size: int):
        packed = _native().table(pages, lens, free, state, page_size)
        for name, value in zip(self.__slots__, (pages, lens, free, state, page_size, packed)):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):      # (the packed structure holds the tensors' addresses)
        raise AttributeError(f"{name} of a PageTable stays what it is")

    @classmethod
    def empty(cls, max_seqs: int, max_pages: int, page_size: int, n_pages: int, device=0) -> "PageTable":
        make = lambda *shape: torch.empty(shape, dtype=torch.int32, device=_cuda(device))
        table = cls(make(max_seqs, max_pages), make(max_seqs), make(n_pages), make(4), page_size)
        table.reset()
        return table

    def reset(self) -> None:
        _native().reset(*self.packed)

    def check(self) -> None:
        """Raises what the status word holds (waits for the stream)."""
        status = int(self.state[1])
        if status != qc.QC_OK:
            raise qc.QcError(status, "page table")


def table_extend(table: PageTable, n_new: Optional[torch.Tensor] = None, *, seq_ids: Optional[torch.Tensor] = None,
                 n_seqs: Optional[int] = None, max_slots: Optional[int] = None):
    """``n_new[i]`` (None: 1) more tokens for row ``seq_ids[i]`` (None: i).  Returns (starts [n + 1], slots [max_slots]):
    sequence i's new tokens are ``starts[i]`` to ``starts[i + 1] - 1`` of the call, token t goes to ``slots[t]``, and slots
    behind the last token are -1.  ``max_slots`` may be left out where every sequence takes one token.  A list without sequences
    changes nothing, here and below."""
    return _native().extend(*table.packed, n_new, seq_ids, n_seqs, max_slots, table.lens)


def table_trim(table: PageTable, n_keep: Optional[torch.Tensor] = None, *, seq_ids: Optional[torch.Tensor] = None,
               n_seqs: Optional[int] = None) -> None:
    """Row ``seq_ids[i]`` (None: i) keeps its first ``n_keep[i]`` tokens (None: none, the sequence is released)."""
    _native().trim(*table.packed, n_keep, seq_ids, n_seqs)


def page_bytes(n_kv_heads: int, head_dim: int, page_size: int) -> int:
    return qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, 1))


def empty_pool(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, device=0) -> torch.Tensor:
    """A pool for one tensor (K or V) of one layer and stream: uint8 [n_pages, page bytes], not initialised."""
    size = qc.qc_quant_pool_bytes(qc.qc_quant_shape(n_kv_heads, head_dim, page_size, n_pages))
    return torch.empty((n_pages, size // n_pages), dtype=torch.uint8, device=_cuda(device))


def append(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, k: Optional[torch.Tensor],
           v: Optional[torch.Tensor], page_size: int) -> None:
    """Quantises rows ``k``, ``v`` (bf16 [tokens, heads, head_dim]; heads dense, tokens any stride that is a multiple of 8)
    into the pools at ``slots``; negative slots are left out.  Either pair may be None (a lazy layer that stores no K)."""
    _native().append(k_pool, v_pool, slots, k, v, page_size)


def read(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, n_kv_heads: int, head_dim: int,
         page_size: int, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """What the rows at ``slots`` stand for: (k, v), bf16 [tokens, n_kv_heads, head_dim], None for a pool that is None.
    Rows of negative slots stay what they were in ``k_out`` / ``v_out`` (zeros where those are made here)."""
    return _native().read(k_pool, v_pool, slots, n_kv_heads, head_dim, page_size, k_out, v_out)


class Stream(NamedTuple):
    """One stream of a cache as ``attend`` reads it: the queries that score its keys (bf16 [tokens, query heads, head_dim]),
    its pools, its table's pages and lengths."""

    q: torch.Tensor
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    pages: torch.Tensor
    lens: torch.Tensor


def attend(text: Stream, n_kv_heads: int, page_size: int, *, visual: Optional[Stream] = None, seq_ids: Optional[torch.Tensor] = None,
           starts: Optional[torch.Tensor] = None, max_queries: int = 1, causal: bool = True, scale: float = 0.0,
           out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Attention of each sequence's query tokens over its cached rows, the queries' own among them (``qc_quant_attend``):
    one softmax over the visual stream's keys, scored by ``visual.q``, and the text stream's, scored by ``text.q``.
    Sequence i is row ``seq_ids[i]`` (None: i) of the tables and has query tokens ``starts[i]`` to ``starts[i + 1] - 1`` (None:
    token i), ``max_queries`` at most.  ``causal``: they are the last tokens of the text stream, and none sees what is behind
    it.  Returns (out bf16 [tokens, query heads, head_dim], lse fp32 [tokens, query heads]); a query that sees nothing gets 0
    and minus infinity; tokens of no sequence stay what they were in ``out`` (where it is made here, anything).
    ``out`` may be a stream's ``q`` itself (dense); it may not overlap one in another way, nor any other argument.  ``status``: an int32 word for what is met on the device (a ``PageTable``'s ``state[1:2]``)."""
    return _native().attend(text, n_kv_heads, page_size, visual, seq_ids, starts, max_queries, causal, scale, out, status)
