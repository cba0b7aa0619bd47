"""Serving from a paged key/value cache held in 4 or in 8 bits: what a decoding loop calls between the model's projections.

    p = CacheParams(H=8, d=128)                              # key/value heads, head dimension; block=64: 8 bits
    cache = alloc_cache(p, pages=4096)
    plan = sagebwd_cache_plan(held, added, block_table, free_pages, free_count, p, rows)   # pages, slots, positions
    Q, K = sage_rotary(Q, K, plan.positions, inv_freq)                                      # (autograd.py)
    sagebwd_cache_append(K, V, plan.slots, cache, p)
    O, LSE = sagebwd_cache_attention(Q, cache, block_table, plan.lengths, plan.cu_new, p, max_new=1)

Requests that share pages (samples of one prompt, the beams of a search):

    shares = alloc_shares(pages=4096)                        # holders of each page
    sagebwd_cache_fork(parents, lengths, block_table, free_pages, free_count, shares, p)    # go on from another request's tokens
    added = sagebwd_cache_own(added, lengths, block_table, free_pages, free_count, shares, cache, p)    # before each plan
    sagebwd_cache_free(keep, lengths, block_table, free_pages, free_count, shares, p)       # in place of trim

Tensors are packed: Q is bf16 [tokens, query heads, d], K and V are bf16 [tokens, H, d], the requests' new tokens one after the other.
They may be slices of one projection's output (adjacent channels, strides that are multiples of 8, rows that begin on 16 bytes).
Formats, arithmetic and bounds of device data: include/sagebwd_serve.h.  Like the calls of `binding`, these are not differentiable,
run on the current stream of their tensors' device, and raise where the library is missing or refuses.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import NamedTuple

import torch

from . import binding

EXPORTS = ("sagebwd_cache_page_bytes", "sagebwd_cache_plan", "sagebwd_cache_trim", "sagebwd_cache_append", "sagebwd_cache_read",
           "sagebwd_cache_workspace_bytes", "sagebwd_cache_attention", "sagebwd_rotary", "sagebwd_cache_free", "sagebwd_cache_fork",
           "sagebwd_cache_fork_workspace_bytes", "sagebwd_cache_own", "sagebwd_cache_compact", "sagebwd_cache_compact_workspace_bytes")


class _CCacheParams(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("d", ctypes.c_int32), ("page", ctypes.c_int32), ("group", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("block", ctypes.c_int32)]


@dataclass
class CacheParams:
    H: int              # key/value heads
    d: int              # 64 or 128
    page: int = 64      # tokens of a page: 32, 64, 128 or 256
    group: int = 64     # channels that share a scale: 32 (4.5 bits a value) or 64 (4.25)
    block: int = 0      # 0: held in 4 bits; 32 or 64: in 8, tokens of a head that share a scale (`group` is not looked at then)


class CachePlan(NamedTuple):
    slots: torch.Tensor      # int64 [rows]: where each new token goes, -1 for none
    positions: torch.Tensor  # int32 [rows]: its place in its request
    cu_new: torch.Tensor     # int32 [R + 1]: where each request's new tokens begin
    lengths: torch.Tensor    # int32 [R]: tokens after the step
    granted: torch.Tensor    # int32 [R]: 0 where a request got nothing (no pages left, sizes out of range, rows full)
    free_left: torch.Tensor  # int32 [1]: pages left on the stack


def cache_page_bytes(p: CacheParams) -> int:
    """Bytes of a page over all heads."""
    n = ctypes.c_size_t(0)
    cp = _CCacheParams(p.H, p.d, p.page, 0 if p.block else p.group, 1, p.block)
    binding._check(binding.load_library().sagebwd_cache_page_bytes(ctypes.byref(cp), ctypes.byref(n)), "sagebwd_cache_page_bytes")
    return int(n.value)


def alloc_cache(p: CacheParams, pages: int, device="cuda"):
    """A pool: uint8 [pages, H, bytes of a page and head].  What it holds before tokens are appended reaches no result."""
    return torch.empty((pages, p.H, cache_page_bytes(p) // p.H), dtype=torch.uint8, device=device)


def sagebwd_cache_plan(held, added, block_table, free_pages, free_count, p: CacheParams, rows: int, out=None) -> CachePlan:
    """Pages, slots and positions of a step's new tokens (int32 device tensors; `rows` >= all new tokens, or the requests behind
    are not granted; at most 2^30).  block_table [R, columns] gets the granted pages; everything else is in the plan, whose tensors `out` (a
    CachePlan) may bring: `out.lengths` may be `held` and `out.free_left` may be `free_count`.

    Requests are served in order: behind one for which there are not enough pages none that needs a page is granted (trim gives pages
    back, and the next plan may grant them).  A request that is not granted keeps its length; its rows have slot -1."""
    return CachePlan._make(binding._host().cache_plan(held, added, block_table, free_pages, free_count, p.page, rows, out))


def sagebwd_cache_trim(keep, lengths, block_table, free_pages, free_count, p: CacheParams) -> None:
    """Requests keep their first keep[r] tokens (0: done); freed pages go back on the stack.  In place."""
    binding._host().cache_trim(keep, lengths, block_table, free_pages, free_count, p.page)


class CacheCompaction(NamedTuple):
    block_table: torch.Tensor  # int32 [R, columns]: the pages' new numbers
    free_pages: torch.Tensor   # int32 [pages]: the stack, the lowest on top
    free_count: torch.Tensor   # int32 [1]
    shares: torch.Tensor       # int32 [3, pages]
    used: torch.Tensor         # int32 [1]: pages in use, which are 0 .. used - 1


def alloc_shares(pages: int, device="cuda"):
    """The holders of a pool's pages, int32 [3, pages]: row 0 has those beyond a page's first, the others are the calls' own.  Zeros at the start."""
    return torch.zeros((3, pages), dtype=torch.int32, device=device)


def sagebwd_cache_free(keep, lengths, block_table, free_pages, free_count, shares, p: CacheParams) -> None:
    """`sagebwd_cache_trim` where requests share pages: a page goes back on the stack when its last holder gives it up.  In place."""
    binding._host().cache_free(keep, lengths, block_table, free_pages, free_count, shares, p.page)


def sagebwd_cache_fork(parents, lengths, block_table, free_pages, free_count, shares, p: CacheParams) -> None:
    """Request r goes on from what request parents[r] holds (int32; itself, or any number that is no request's: as it is) and gives up what it
    held.  The pages are shared and nothing is copied: `sagebwd_cache_own` does that where a request writes.  In place."""
    binding._host().cache_fork(parents, lengths, block_table, free_pages, free_count, shares, p.page)


def sagebwd_cache_own(added, lengths, block_table, free_pages, free_count, shares, cache, p: CacheParams, out=None):
    """Before a step's plan: a request that is about to add tokens to a page which others hold gets a copy of it from the stack.  Returns added
    (int32 [R]), with 0 for a request that wanted a page when none was left: what the plan is given.  Everything else in place."""
    return binding._host().cache_own(added, lengths, block_table, free_pages, free_count, shares, cache, p.H, p.d, p.page, p.group, p.block, out)


def sagebwd_cache_compact(lengths, block_table, cache, p: CacheParams, out=None) -> CacheCompaction:
    """Moves the pages in use to the front of the pool (in place) and returns the table that names them there, with the stack and shares that go
    with it.  `out` (a CacheCompaction) may bring their tensors, the inputs' own among them; what no row of the table names is free afterwards."""
    return CacheCompaction._make(binding._host().cache_compact(lengths, block_table, cache, p.H, p.d, p.page, p.group, p.block, out))


def sagebwd_cache_append(K, V, slots, cache, p: CacheParams, k_mean=None, v_mean=None) -> None:
    """New keys and values into the cache; k_mean, v_mean: float32 [H, d], taken off before they are quantised (one for all tokens: a model's,
    with which the whole pool is filled).  Held in 8 bits, a block's scale grows with its tokens, whose codes are then written again: the tokens
    of a block that a call brings stand one after the other, their slots rising by one (as a plan has them)."""
    binding._host().cache_append(K, V, slots, cache, p.H, p.d, p.page, p.group, p.block, k_mean, v_mean)


def sagebwd_cache_read(slots, cache, p: CacheParams, k_mean=None, v_mean=None, K=None, V=None):
    """(K, V) bf16 [tokens, H, d]: the values that the cache holds at `slots` (zeros for -1), exactly (held in 8 bits: rounded); with means,
    value + mean in float32, rounded."""
    return binding._host().cache_read(slots, cache, p.H, p.d, p.page, p.group, p.block, k_mean, v_mean, K, V)


def cache_workspace_bytes(p: CacheParams, R: int, T: int, Hq: int, columns: int, max_new: int, max_length: int = 0) -> int:
    """Bytes of workspace of `sagebwd_cache_attention` for R requests, T rows of Hq query heads and that many table columns."""
    return binding._host().cache_workspace_bytes(p.H, p.d, p.page, p.group, p.block, R, T, Hq, columns, max_new, max_length)


def sagebwd_cache_attention(Q, cache, block_table, lengths, cu, p: CacheParams, max_new: int, causal: bool = True, sm_scale: float = 0.0,
                            v_mean=None, max_length: int = 0, workspace=None, O=None, LSE=None):
    """O bf16 [tokens, query heads, d] and LSE float32 [query heads, tokens] of every request's new tokens over its cache.

    `max_new` and `max_length` (0: whatever the table holds) bound the requests' new tokens and lengths on the host: how the call is laid out and
    its workspace go by them, so that a table wider than the requests are long wants a `max_length`.  Rows behind the last request are left as
    they are in O and LSE.  A row that sees no key has O = 0 and LSE = -infinity."""
    return binding._host().cache_attention(Q, cache, block_table, lengths, cu, p.H, p.d, p.page, p.group, p.block, max_new, causal, sm_scale, v_mean,
                                           max_length, workspace, O, LSE)
