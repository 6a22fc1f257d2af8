"""Serving steps that need no host in between: pages handed out on the device, and the choice of blocks of the far past for the heads
that read it - the Python names of ``seg_pages_resize``, ``seg_blocks_summarise`` and ``seg_blocks_select``.

A decoding step is then ``pages_resize`` (lengths, block table, positions), ``kv_append`` (which with scales of blocks keeps an
8-bit cache's scales itself), ``blocks_summarise`` (means of the blocks that have become full), ``blocks_select`` and
``seg_attn_decode(..., blocks=...)``, all on one stream, and can be captured in a CUDA graph as a whole.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import lib
from .paged import _CACHE, _F32, _I32, _block_scales, _cache, _call, _flat, _mask_bytes, _on_stream, _p, _pages, _rows4

_MEANS = struct.Struct("2Pi4x")        # seg_block_means


@_on_stream
def pages_resize(want, block_table, kv_len, free_pages, free_count, page_size: int, Lq: int, pos_shift: Optional[torch.Tensor] = None,
                 kv_len_out=None, free_count_out=None, q_len=None, slots=None, positions=None, workspace: Optional[torch.Tensor] = None,
                 stream=None):
    """Brings every sequence to the length `want` (int32 [B]): pages behind it go back to the list free_pages (int32 [n_pages], the
    first free_count (int32 [1]) of them free), and sequences that grow (by up to Lq rows) take pages from its end, in order, until there are not
    enough: those stay as they are - the C entry point `seg_pages_resize`.  block_table [B, max_pages] gets the new entries.
    Returns (kv_len_out, free_count_out, q_len, slots, positions): the lengths (kv_len_out may be kv_len or want), the list's new length (may be
    free_count), the new rows of every sequence, and for each of them, [B, Lq], its row in the pages taken as one (int64, -1: not there) and
    its position (int32, pos_shift added).  kv_append takes the lengths and the new rows (kv_len, q_len) and finds their places by itself;
    rope_rotate takes the positions; the slot map is for kernels of a program's own that write beside the cache."""
    dev = want.get_device()
    if dev < 0:
        raise ValueError("pages are handed out on a CUDA device: want and the others lie there")
    B, per, stride = _pages(block_table, None, "block_table", dev)
    _flat(want, _I32, (B,), "want", dev)
    _flat(kv_len, _I32, (B,), "kv_len", dev)
    if free_pages.dim() != 1:
        raise ValueError("free_pages must be an int32 tensor [n_pages]")
    n_pages = free_pages.shape[0]
    _flat(free_pages, _I32, (n_pages,), "free_pages", dev)
    _flat(free_count, _I32, (1,), "free_count", dev)
    if pos_shift is not None:
        _flat(pos_shift, _I32, (B,), "pos_shift", dev)
    kv_len_out = torch.empty_like(kv_len) if kv_len_out is None else _flat(kv_len_out, _I32, (B,), "kv_len_out", dev)
    free_count_out = torch.empty_like(free_count) if free_count_out is None else _flat(free_count_out, _I32, (1,), "free_count_out", dev)
    q_len = torch.empty_like(kv_len) if q_len is None else _flat(q_len, _I32, (B,), "q_len", dev)
    rows = (B, max(Lq, 0))
    slots = want.new_empty(rows, dtype=torch.int64) if slots is None else _flat(slots, torch.int64, rows, "slots", dev)
    positions = want.new_empty(rows) if positions is None else _flat(positions, _I32, rows, "positions", dev)
    L = lib()
    if workspace is None:
        if B > 1024 or B * Lq > 4096:      # smaller calls need none
            workspace = torch.empty(max(L.seg_pages_workspace_bytes(B), 256), dtype=torch.uint8, device=want.device)
    elif workspace.get_device() != dev:
        raise ValueError("workspace must be on the tables' device")
    _call(dev, stream, L.seg_pages_resize, "seg_pages_resize", B, Lq, page_size, n_pages, want.data_ptr(), block_table.data_ptr(), per, stride,
          kv_len.data_ptr(), _p(pos_shift), free_pages.data_ptr(), free_count.data_ptr(), kv_len_out.data_ptr(), free_count_out.data_ptr(),
          q_len.data_ptr(), slots.data_ptr(), positions.data_ptr(), _p(workspace), workspace.nbytes if workspace is not None else 0)
    return kv_len_out, free_count_out, q_len, slots, positions


def _means(sums, sum_scale, page_size: int, dev: int):
    """seg_block_means as bytes, and (n_pages, Hkv, d)."""
    if sums.dim() != 4 or sums.dtype is not torch.int8 or sums.get_device() != dev or not sums.is_contiguous():
        raise ValueError("sums must be a contiguous int8 tensor [n_pages, blocks of a page, Hkv, d] on CUDA device %d" % dev)
    n_pages, per, Hkv, d = sums.shape
    _flat(sum_scale, _F32, (n_pages, per, Hkv), "sum_scale", dev)
    if per < 1 or page_size % per:
        raise ValueError("a page has a whole number of blocks: sums is [n_pages, page_size / block, Hkv, d]")
    return _MEANS.pack(sums.data_ptr(), sum_scale.data_ptr(), page_size // per), n_pages, Hkv, d


@_on_stream
def blocks_summarise(K_pages, block_table, kv_len, Lq: int, sums, sum_scale, q_len: Optional[torch.Tensor] = None, k_scale=None, stream=None):
    """Mean keys of the blocks that hold one of the newest q_len (None: Lq) rows of a sequence and are full (and of those that share a
    scale's block with such a row, whose rows the append may have rounded anew), into sums (int8
    [n_pages, page_size / block, Hkv, d]) times sum_scale (fp32 [n_pages, page_size / block, Hkv]) - the C entry point
    `seg_blocks_summarise`.  kv_len counts the new rows already; to rebuild all means, pass Lq = max_pages * page_size."""
    dev = K_pages.get_device()
    sc = _block_scales(k_scale, k_scale, K_pages, dev)
    one = k_scale if sc is None else None
    c, _, Hkv, d, page, _, dev = _cache(K_pages, K_pages, block_table, kv_len, q_len, None, one, one, reads_values=sc is None)
    m, n_pages, heads, width = _means(sums, sum_scale, page, dev)
    if (n_pages, heads, width) != (K_pages.shape[0], Hkv, d):
        raise ValueError("sums must be [n_pages, page_size / block, Hkv, d] of the cache's pages")
    _call(dev, stream, lib().seg_blocks_summarise, "seg_blocks_summarise", c, sc, Lq, m)


@_on_stream
def blocks_select(Q, sums, sum_scale, block_table, kv_len, page_size: int, S: int, T: int, n: int, sink: int = 0, head_past_mask=None,
                  q_len: Optional[torch.Tensor] = None, pos_shift: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  stream=None):
    """int32 [B, Lq, Hkv, n]: for each new row Q [B, Lq, Hq, d] and KV head with its past (class 1) the blocks in front of its
    segment's tail (segments of S, tail T) whose means score highest against the head's summed queries, the first `sink` blocks in any case,
    ascending and filled up with -1 - the C entry point `seg_blocks_select`.  seg_attn_decode takes it as `blocks`."""
    dev = Q.get_device()
    if Q.dim() != 4:
        raise ValueError("Q must be [B, Lq, Hq, d]")
    m, n_pages, Hkv, d = _means(sums, sum_scale, page_size, dev)
    B, per, stride = _pages(block_table, None, "block_table", dev)
    Lq, Hq = Q.shape[1], Q.shape[2]
    qs = _rows4(Q, (B, Lq, Hq, d), "Q", dev)
    _flat(kv_len, _I32, (B,), "kv_len", dev)
    if q_len is not None:
        _flat(q_len, _I32, (B,), "q_len", dev)
    if pos_shift is not None:
        _flat(pos_shift, _I32, (B,), "pos_shift", dev)
    out = Q.new_empty((B, Lq, Hkv, max(n, 0)), dtype=_I32) if out is None else _flat(out, _I32, (B, Lq, Hkv, n), "out", dev)
    c = _CACHE.pack(B, Hkv, d, 0, page_size, n_pages, per, stride, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, block_table.data_ptr(), kv_len.data_ptr(),
                    _p(q_len) or 0, _p(pos_shift) or 0)
    _call(dev, stream, lib().seg_blocks_select, "seg_blocks_select", c, Lq, Hq, S, T, _mask_bytes(head_past_mask, Hkv), Q.data_ptr(), qs, m, n, sink,
          out.data_ptr())
    return out
