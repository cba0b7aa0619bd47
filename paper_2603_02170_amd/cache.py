"""Serving from a paged key/value cache held in 4 bits: what a decoding loop calls between the model's projections.

    p = CacheParams(H=8, d=128)                              # key/value heads, head dimension
    cache = alloc_cache(p, pages=4096)
    plan = sagebwd_cache_plan(held, added, block_table, free_pages, free_count, p, rows)   # pages, slots, positions
    Q, K = sage_rotary(Q, K, plan.positions, inv_freq)                                      # (autograd.py)
    sagebwd_cache_append(K, V, plan.slots, cache, p)
    O, LSE = sagebwd_cache_attention(Q, cache, block_table, plan.lengths, plan.cu_new, p, max_new=1)

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
           "sagebwd_cache_workspace_bytes", "sagebwd_cache_attention", "sagebwd_rotary")


class _CCacheParams(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("d", ctypes.c_int32), ("page", ctypes.c_int32), ("group", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("reserved", ctypes.c_int32)]


@dataclass
class CacheParams:
    H: int              # key/value heads
    d: int              # 64 or 128
    page: int = 64      # tokens of a page: 32, 64, 128 or 256
    group: int = 64     # channels that share a scale: 32 (4.5 bits a value) or 64 (4.25)


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
    cp = _CCacheParams(p.H, p.d, p.page, p.group, 1, 0)
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


def sagebwd_cache_append(K, V, slots, cache, p: CacheParams, k_mean=None, v_mean=None) -> None:
    """New keys and values into the cache; k_mean, v_mean: float32 [H, d], taken off before they are quantised (one for all tokens: a model's,
    with which the whole pool is filled)."""
    binding._host().cache_append(K, V, slots, cache, p.H, p.d, p.page, p.group, k_mean, v_mean)


def sagebwd_cache_read(slots, cache, p: CacheParams, k_mean=None, v_mean=None, K=None, V=None):
    """(K, V) bf16 [tokens, H, d]: the values that the cache holds at `slots` (zeros for -1), exactly; with means, value + mean in float32,
    rounded."""
    return binding._host().cache_read(slots, cache, p.H, p.d, p.page, p.group, k_mean, v_mean, K, V)


def cache_workspace_bytes(p: CacheParams, R: int, T: int, Hq: int, columns: int, max_new: int, max_length: int = 0) -> int:
    """Bytes of workspace of `sagebwd_cache_attention` for R requests, T rows of Hq query heads and that many table columns."""
    return binding._host().cache_workspace_bytes(p.H, p.d, p.page, p.group, R, T, Hq, columns, max_new, max_length)


def sagebwd_cache_attention(Q, cache, block_table, lengths, cu, p: CacheParams, max_new: int, causal: bool = True, sm_scale: float = 0.0,
                            v_mean=None, max_length: int = 0, workspace=None, O=None, LSE=None):
    """O bf16 [tokens, query heads, d] and LSE float32 [query heads, tokens] of every request's new tokens over its cache.

    `max_new` and `max_length` (0: whatever the table holds) bound the requests' new tokens and lengths on the host: how the call is laid out and
    its workspace go by them, so that a table wider than the requests are long wants a `max_length`.  Rows behind the last request are left as
    they are in O and LSE.  A row that sees no key has O = 0 and LSE = -infinity."""
    return binding._host().cache_attention(Q, cache, block_table, lengths, cu, p.H, p.d, p.page, p.group, max_new, causal, sm_scale, v_mean,
                                           max_length, workspace, O, LSE)
