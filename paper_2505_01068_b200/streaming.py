"""A stream's past in 8 bits: caches of keys and values, and the calls of gsit_stream.h on them.

A step of a batch of streams is cache_plan (where do its rows go?), cache_append (its keys and values) and im_cached_attention_fwd (its queries against
all that is held then), or cache_step, which is all three.  Lengths, tables and counts stay on the device, so a step can be captured into a graph and replayed."""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B

CACHE_BLOCK = 32   # positions of a block, a scale each for every key head


class StreamTables(NamedTuple):
    """Where blocks lie: tables int32 [B, 3, blocks] (page of each block of a segment, -1: none), lengths int32 [B, 3] (positions held), free int32
    [pages] with n_free int32 [1] of them in use (pages that no block has)."""
    tables: torch.Tensor
    lengths: torch.Tensor
    free: torch.Tensor
    n_free: torch.Tensor


class StreamCache(NamedTuple):
    """StreamTables and what lies there: keys and values int8 or float8_e4m3fn [pages, Hk, 32 * hd] (in the order that gsit_stream.h gives), their scales float32
    [pages, Hk], times float32 [pages, 32] or None, and the rows of blocks that are not full, [B, 3, 2, Hk, 32, hd]."""
    tables: torch.Tensor
    lengths: torch.Tensor
    free: torch.Tensor
    n_free: torch.Tensor
    times: Optional[torch.Tensor]
    keys: torch.Tensor
    values: torch.Tensor
    key_scale: torch.Tensor
    value_scale: torch.Tensor
    open_keys: torch.Tensor
    open_values: torch.Tensor


def stream_tables(batch, blocks, pages, device="cuda"):
    """Tables of streams that hold nothing, `blocks` blocks to a segment at most, over a pool of `pages` pages."""
    return StreamTables(torch.full((batch, 3, blocks), -1, dtype=torch.int32, device=device), torch.zeros((batch, 3), dtype=torch.int32, device=device),
                        torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device), torch.full((1,), pages, dtype=torch.int32, device=device))


def stream_cache(batch, max_len, kv_heads, head_dim, dtype=torch.bfloat16, held_as="int8", pages=None, times=False, device="cuda"):
    """An empty cache for `batch` streams of at most max_len (three numbers) positions a segment, held as "int8" or "e4m3"; pages: of the pool (default: enough
    for all streams at their longest).  times: every position has a moment (causality and slopes go by it).  head_dim 8, 16, 32 or 64; dtype float32 or bfloat16."""
    if held_as not in ("int8", "e4m3"):
        raise ValueError('held_as: "int8" or "e4m3"')
    if head_dim not in (8, 16, 32, 64) or dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("a cache holds heads of 8, 16, 32 or 64 features, float32 or bfloat16")
    need = [(int(n) + CACHE_BLOCK - 1) // CACHE_BLOCK for n in max_len]
    pages = max(1, batch * sum(need)) if pages is None else int(pages)
    zeros = lambda shape, t: torch.zeros(shape, dtype=t, device=device)
    t8 = torch.int8 if held_as == "int8" else torch.float8_e4m3fn
    page, scale, opened = (pages, kv_heads, CACHE_BLOCK * head_dim), (pages, kv_heads), (batch, 3, 2, kv_heads, CACHE_BLOCK, head_dim)
    return StreamCache(*stream_tables(batch, max(1, *need), pages, device), zeros((pages, CACHE_BLOCK), torch.float32) if times else None,
                       zeros(page, torch.uint8).view(t8), zeros(page, torch.uint8).view(t8), zeros(scale, torch.float32), zeros(scale, torch.float32),
                       zeros(opened, dtype), zeros(opened, dtype))


def cache_plan(cache, seg_len, valid_len=None, ended=None, held=None, slots=None):
    """Pages for a step that brings valid_len [B, 3] (default: seg_len) rows, and the slot int32 [B, L] of each: 32 * page + place, -1 for padding.  Updates
    tables, lengths (held + valid_len; held int32 [B, 3], default: lengths) and the list of free pages.  ended int32 [B]: streams other than 0 begin
    anew.  What finds no room is left out (slots -1) and raises DEVFLAG_FULL in last_device_status."""
    return B.native().cache_plan(cache.tables, cache.lengths, cache.free, cache.n_free, seg_len, valid_len, ended, held, slots)


def cache_append(cache, k, v, slots, seg_len, times=None):
    """The step's keys and values [B, L, Hk, hd] into the cache, where cache_plan, called with the same seg_len, said; times float32 [B, L] where the cache
    holds them."""
    B.native().cache_append(*cache, k, v, slots, seg_len, times)


def cache_read(cache, seg_len, out_k=None, out_v=None):
    """(k, v) [B, L, Hk, hd]: the first seg_len positions of every segment as rows, +0 behind the last one held."""
    return B.native().cache_read(*cache, seg_len, out_k, out_v)


def im_cached_attention_fwd(q, cache, seg_len, valid_len=None, phase=B.PHASE_INTER_FWD, custom_mask=0, scale=0.0, softcap=0.0, slopes=None, times=None, causal=False,
                            want_lse=False, out=None, workspace=None):
    """im_scored_attention_fwd for a step's rows q [B, L, H, hd] against the cache: real row i of segment s is position lengths - valid_len + i of it.
    times float32 [B, L]: moments of these rows, where the cache holds moments (None where it does not: the index inside the segment, in tables of
    at most 2^19 blocks).  Returns out [B, L, d] (and lse [B, H, L])."""
    return B.native().cached_attention(*cache, q, seg_len, valid_len, phase, custom_mask, scale, softcap, slopes, times, causal, want_lse, out, workspace)


def cache_step(cache, q, k, v, seg_len, valid_len=None, ended=None, held=None, phase=B.PHASE_INTER_FWD, custom_mask=0, scale=0.0, softcap=0.0, slopes=None, times=None,
               causal=False, slots=None, out=None, workspace=None):
    """cache_plan, cache_append and im_cached_attention_fwd for a step's rows q [B, L, H, hd], k and v [B, L, Hk, hd], in one call that changes nothing of the
    cache where any of the three refuses its arguments.  Returns (out [B, L, d], slots [B, L])."""
    return B.native().cache_step(*cache, q, k, v, seg_len, valid_len, ended, held, phase, custom_mask, scale, softcap, slopes, times, causal, slots, out, workspace)
