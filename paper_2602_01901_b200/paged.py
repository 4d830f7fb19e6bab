"""What stands between a projection and its attention, and a K/V cache in bf16 pages on the device's page tables.

The calls of ``include/qc.h`` on torch tensors, in the manner of ``quant``: every buffer is the caller's, every call is
enqueued on the current stream of the tensors' device and returns at once, nothing is kept between calls, so a step can be
captured into a ``torch.cuda.graph`` and replayed.  ``ValueError`` and ``QcError`` for arguments that do not fit.  Page tables
are ``quant``'s: their slots do for both kinds of cache.  No gradient flows through any of the calls.

    rotation = Rotation(freqs, axes)                                                           # of the model
    q, k = rotate(q, k, positions, rotation, q_norm=wq, k_norm=wk)                             # for any cache: rotated rows
    table = PageTable.empty(max_seqs, max_pages, page_size, n_pages)
    k_pool, v_pool = (empty_pool(n_kv_heads, head_dim, page_size, n_pages) for _ in "kv")      # of each layer
    starts, slots = table_extend(table, n_new, seq_ids=ids, max_slots=n_tokens)                # once a step
    q = append(k_pool, v_pool, slots, k, v, q=q, positions=positions, rotation=rotation)       # each layer
    out, lse = attend(Stream(q, k_pool, v_pool, table.pages, table.lens), seq_ids=ids, starts=starts, max_queries=most,
                      shared=Stream(q, k_image, v_image, images.pages, images.lens), groups=groups, shared_ids=image_ids)
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from .quant import PageTable, Stream, _cuda, _native, table_extend, table_trim  # noqa: F401  (the tables of both caches)


class Rotation(NamedTuple):
    """How pairs of elements are turned: pair i by ``positions[axes[i]] * freqs[i]`` radians.  ``freqs``: float32 [pairs] on the device, a
    multiple of 8 pairs; the first 2 * pairs elements of a head are turned, the others pass.  ``axes``: int32 [pairs], None: all
    the first axis.  Pairs are elements (i, i + pairs), or (2 i, 2 i + 1) where ``adjacent``."""

    freqs: torch.Tensor
    axes: Optional[torch.Tensor] = None
    adjacent: bool = False


def rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor], rotation: Optional[Rotation], *,
           q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Rows of ``q`` and ``k`` (bf16 [tokens, heads, head_dim]; heads dense, tokens any stride that is a multiple of 8; either may
    be None) divided by their root mean square and times the weights where ``q_norm`` / ``k_norm`` (bf16 or float32 [head_dim]) are
    given, then turned by ``positions`` (int32 [tokens] or [axes, tokens]) where there is a ``rotation``.  Returns (q, k).  An output
    may be its own input, in place."""
    return _native().rotate(q, k, positions, rotation, q_norm, k_norm, eps, q_out, k_out)


def empty_pool(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, device=0) -> torch.Tensor:
    """A pool for one tensor (K or V) of one layer and stream: bf16 [n_pages, n_kv_heads, page_size, head_dim], not initialised."""
    return torch.empty((n_pages, n_kv_heads, page_size, head_dim), dtype=torch.bfloat16, device=_cuda(device))


def append(k_pool: Optional[torch.Tensor], v_pool: Optional[torch.Tensor], slots: torch.Tensor, k: Optional[torch.Tensor],
           v: Optional[torch.Tensor], *, q: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
           rotation: Optional[Rotation] = None, q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None,
           eps: float = 1e-6, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Stores rows ``k``, normalised and turned as by ``rotate``, and ``v`` as they are at ``slots``; negative slots are left out.  Either
    pair of pool and rows may be None (a lazy layer that stores no K).  Returns ``q``'s rows as ``rotate`` makes them, of all tokens
    (None without ``q``)."""
    return _native().paged_append(k_pool, v_pool, slots, k, v, q, positions, rotation, q_norm, k_norm, eps, q_out)


def attend(own: Stream, *, shared: Optional[Stream] = None, groups: Optional[torch.Tensor] = None, shared_ids: Optional[torch.Tensor] = None,
           seq_ids: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None, max_queries: int = 1, causal: bool = True,
           scale: float = 0.0, out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Attention of each sequence's query tokens over the prefix that its group shares and its own cached rows, the queries' own among
    them (``qc_paged_attend``): one softmax over the prefix's keys, scored by ``shared.q``, and its own, scored by ``own.q``.  Sequence i
    is row ``seq_ids[i]`` (None: i) of the own table and has query tokens ``starts[i]`` to ``starts[i + 1] - 1`` (None: token i),
    ``max_queries`` at most.  Sequences ``groups[g]`` to ``groups[g + 1] - 1`` share row ``shared_ids[g]`` (None: g) of the shared
    stream's table (``groups`` None: all share one); sequences before and behind the groups have no prefix.  A prefix is read
    once for its group.  ``causal``: the queries are the last tokens of their own stream, and none sees what is behind it.  Returns
    (out bf16 [tokens, query heads, head_dim], lse fp32 [tokens, query heads]); scores and sums are fp32, weights are rounded to bf16 for their
    products with values; a query that sees nothing gets 0 and minus infinity; tokens
    of no sequence stay what they were in ``out`` (where it is made here, anything).  ``out`` overlaps no other argument.  ``status``: an
    int32 word for what is met on the device (a ``PageTable``'s ``state[1:2]``): lists that do not fit, or too much work for a call, leave ``out`` as it
    was, and only this word says so."""
    return _native().paged_attend(own, shared, groups, shared_ids, seq_ids, starts, max_queries, causal, scale, out, status)
