"""Serving from a paged key/value cache, and rotary positions in general form: the Python names of the C entry points
``seg_kv_append``, ``seg_attn_decode``, ``seg_kv_evict``, ``seg_rope_table_scaled`` and ``seg_rope_rotate``.

A cache is described by the same tensors in every call:

``K_pages``, ``V_pages``  ``[n_pages, page_size, Hkv, d]``, bf16 or ``torch.float8_e4m3fn``; any strides that are multiples
                          of 16 bytes with a contiguous last dimension (a permuted ``[n_pages, Hkv, page_size, d]`` buffer too)
``block_table``           int32 ``[B, max_pages]``: the pages of every sequence in order
``kv_len``                int32 ``[B]``: rows of every sequence, the call's new ones included
``q_len``                 int32 ``[B]`` or None: how many of the ``Lq`` rows given are there (the first ones); None: all
``pos_shift``             int32 ``[B]`` or None: rows that evictions have taken out (global position = slot + shift)
``k_scale``, ``v_scale``  fp32 ``[Hkv]``, for an 8-bit cache only

Lengths stay on the device, so that a decoding step can be captured in a CUDA graph and replayed as they grow.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import SegAttnError, _mask_arr, lib

_CACHE = struct.Struct("8i2P6q6P")     # seg_kv_cache
_STRIDE3 = struct.Struct("3q")
_SCALING = struct.Struct("i4x6d")      # seg_rope_scaling
_LAYOUTS = {"half": 0, "interleaved": 1}
_KINDS = {"plain": 0, "linear": 1, "by_parts": 2}


def _check(status: int, where: str):
    if status != 0:
        raise SegAttnError(status, where)


def _p(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _layout(name) -> int:
    if name not in _LAYOUTS:
        raise ValueError("layout must be 'half' or 'interleaved'")
    return _LAYOUTS[name]


def _rows4(t: torch.Tensor, shape, what: str) -> bytes:
    """The (batch, row, head) strides of a bf16 CUDA tensor of this shape, the last dimension contiguous."""
    if t.dtype is not torch.bfloat16 or not t.is_cuda or t.shape != shape:
        raise ValueError("%s must be a bf16 CUDA tensor of shape %s" % (what, tuple(shape)))
    s = t.stride()
    if s[3] != 1:
        raise ValueError("%s must have a contiguous last dimension" % what)
    return _STRIDE3.pack(s[0], s[1], s[2])


def _flat(t, dtype, shape, what: str, device):
    """A contiguous CUDA tensor of this type and shape on this device, or None."""
    if t is not None and (t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (what, dtype, tuple(shape), device))
    return t


def _on(device, stream):
    """The stream to launch on: the given one, or the tensors' device's current one."""
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        raise ValueError("the stream belongs to another device than the tensors")
    return stream.cuda_stream


def _call(device, fn, where, *args):
    """One C call with the tensors' device current."""
    if torch.cuda.current_device() == device.index:
        _check(fn(*args), where)
    else:
        with torch.cuda.device(device):
            _check(fn(*args), where)


def _cache(K, V, block_table, kv_len, q_len, pos_shift, k_scale, v_scale):
    """seg_kv_cache of these tensors as bytes, and (B, Hkv, d, page_size, max_pages)."""
    dev = K.device
    if K.dim() != 4 or K.shape != V.shape or not K.is_cuda or V.device != dev or K.dtype is not V.dtype:
        raise ValueError("K_pages and V_pages must be CUDA tensors [n_pages, page_size, Hkv, d] of one shape, type and device")
    if K.dtype is torch.bfloat16:
        kind = 0
        if k_scale is not None or v_scale is not None:
            raise ValueError("scales belong to an 8-bit cache")
    elif K.dtype is torch.float8_e4m3fn:
        kind = 1
        if k_scale is None or v_scale is None:
            raise ValueError("an 8-bit cache needs k_scale and v_scale")
    else:
        raise ValueError("the cache must be bf16 or float8_e4m3fn")
    n_pages, page, Hkv, d = K.shape
    ks, vs = K.stride(), V.stride()
    if ks[3] != 1 or vs[3] != 1:
        raise ValueError("the pages must have a contiguous last dimension")
    if block_table.dim() != 2 or block_table.dtype is not torch.int32 or block_table.device != dev or block_table.stride(1) != 1:
        raise ValueError("block_table must be an int32 tensor [B, max_pages] on %s with contiguous rows" % dev)
    B, max_pages = block_table.shape
    if kv_len is None:
        raise ValueError("kv_len is needed")
    for t, what in ((kv_len, "kv_len"), (q_len, "q_len"), (pos_shift, "pos_shift")):
        _flat(t, torch.int32, (B,), what, dev)
    _flat(k_scale, torch.float32, (Hkv,), "k_scale", dev)
    _flat(v_scale, torch.float32, (Hkv,), "v_scale", dev)
    c = _CACHE.pack(B, Hkv, d, kind, page, n_pages, max_pages, max(block_table.stride(0), max_pages) if B > 1 else max_pages,
                    K.data_ptr(), V.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], _p(k_scale) or 0, _p(v_scale) or 0,
                    block_table.data_ptr(), kv_len.data_ptr(), _p(q_len) or 0, _p(pos_shift) or 0)
    if B > 1 and block_table.stride(0) < max_pages:
        raise ValueError("the rows of block_table overlap")
    return c, B, Hkv, d, page, max_pages


def rope_table_scaled(n_pos: int, rot_dim: int, base: float = 10000.0, kind: str = "plain", factor: float = 1.0,
                      trained_len: float = 0.0, turns_lo: float = 0.0, turns_hi: float = 0.0, amplitude: float = 1.0,
                      device="cuda", stream=None) -> torch.Tensor:
    """fp32 [n_pos, rot_dim/2, 2] = amplitude * (cos, sin) of pos * w_i - the C entry point `seg_rope_table_scaled`.
    `kind` "plain": w_i = base^(-2i/rot_dim); "linear": w_i / factor; "by_parts": pairs that make fewer than `turns_lo` turns
    over `trained_len` positions are divided by `factor`, those of more than `turns_hi` kept, a ramp between."""
    if kind not in _KINDS:
        raise ValueError("kind must be 'plain', 'linear' or 'by_parts'")
    if n_pos < 0 or rot_dim < 0:
        raise SegAttnError(1, "seg_rope_table_scaled")
    table = torch.empty((n_pos, rot_dim // 2, 2), dtype=torch.float32, device=device)
    sc = _SCALING.pack(_KINDS[kind], base, factor, trained_len, turns_lo, turns_hi, amplitude)
    _call(table.device, lib().seg_rope_table_scaled, "seg_rope_table_scaled", n_pos, rot_dim, sc, table.data_ptr(),
          _on(table.device, stream))
    return table


def _table(table, device):
    if (table.dim() != 3 or table.shape[2] != 2 or table.dtype is not torch.float32 or table.device != device or
            not table.is_contiguous()):
        raise ValueError("table must be a contiguous fp32 tensor [n_pos, rot_dim/2, 2] on %s" % device)
    return table.shape[0], 2 * table.shape[1]


def rope_rotate(X, table, positions: Optional[torch.Tensor] = None, pos0: int = 0, layout: str = "half", inverse: bool = False,
                out: Optional[torch.Tensor] = None, stream=None):
    """Rows of X [B, L, H, d] rotated at `positions` (int32 [B, L]; None: pos0, pos0 + 1, ...) by a table of rope_table or
    rope_table_scaled, whose width is the part of the head that turns - the C entry point `seg_rope_rotate`.  `layout` names
    the pairs: "half" (x[i], x[i + rot/2]) or "interleaved" (x[2i], x[2i+1]).  inverse=True applies the transposed map, which
    takes the gradient of the output to that of X.  `out` may be X."""
    if X.dim() != 4:
        raise ValueError("X must be [B, L, H, d]")
    xs = _rows4(X, X.shape, "X")
    Y = torch.empty(X.shape, dtype=X.dtype, device=X.device) if out is None else out
    ys = _rows4(Y, X.shape, "out") if out is not None else _STRIDE3.pack(*Y.stride()[:3])
    dev = X.device
    if Y.device != dev:
        raise ValueError("out must be on the device of X")
    if Y.data_ptr() == X.data_ptr() and X.numel() and xs != ys:
        raise ValueError("a rotation in place needs the strides of X")
    n_pos, rot = _table(table, dev)
    B, L, H, d = X.shape
    _flat(positions, torch.int32, (B, L), "positions", dev)
    _call(dev, lib().seg_rope_rotate, "seg_rope_rotate", B, L, H, d, rot, _layout(layout), X.data_ptr(), xs, Y.data_ptr(), ys,
          _p(positions), pos0, int(bool(inverse)), table.data_ptr(), n_pos, _on(dev, stream))
    return Y


def kv_append(K_new, V_new, K_pages, V_pages, block_table, kv_len, table: Optional[torch.Tensor] = None, layout: str = "half",
              Q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, q_len=None, pos_shift=None, k_scale=None,
              v_scale=None, stream=None):
    """New rows K_new, V_new [B, Lq, Hkv, d] into the cache; with a table the keys, and the queries Q [B, Lq, Hq, d] if given,
    are rotated at their positions - the C entry point `seg_kv_append`.  Returns the rotated queries (q_out, which may be Q),
    or None.  kv_len counts the new rows already."""
    c, B, Hkv, d, _, _ = _cache(K_pages, V_pages, block_table, kv_len, q_len, pos_shift, k_scale, v_scale)
    dev = K_pages.device
    if K_new.dim() != 4 or K_new.device != dev or V_new.device != dev:
        raise ValueError("K_new and V_new must be [B, Lq, Hkv, d] on the cache's device")
    Lq = K_new.shape[1]
    kn, vn = _rows4(K_new, (B, Lq, Hkv, d), "K_new"), _rows4(V_new, (B, Lq, Hkv, d), "V_new")
    n_pos = rot = Hq = 0
    if table is not None:
        n_pos, rot = _table(table, dev)
    qs = qo = None
    if Q is not None:
        if table is None:
            raise ValueError("queries are rotated by a table")
        Hq = Q.shape[2] if Q.dim() == 4 else 0
        qs = _rows4(Q, (B, Lq, Hq, d), "Q")
        if q_out is None:
            q_out = torch.empty(Q.shape, dtype=Q.dtype, device=dev)
        qo = _rows4(q_out, (B, Lq, Hq, d), "q_out")
        if Q.device != dev or q_out.device != dev:
            raise ValueError("Q and q_out must be on the cache's device")
        if q_out.data_ptr() == Q.data_ptr() and Q.numel() and qs != qo:
            raise ValueError("a rotation in place needs the strides of Q")
    elif q_out is not None:
        raise ValueError("q_out needs Q")
    _call(dev, lib().seg_kv_append, "seg_kv_append", c, Lq, K_new.data_ptr(), kn, V_new.data_ptr(), vn, Hq, _p(Q), qs, _p(q_out),
          qo, _p(table), n_pos, rot, _layout(layout), _on(dev, stream))
    return q_out


def seg_attn_decode(Q, K_pages, V_pages, block_table, kv_len, S: int, T: int, head_past_mask=None, sm_scale: Optional[float] = None,
                    q_len=None, pos_shift=None, k_scale=None, v_scale=None, weights=None, weights_out=None, out=None, lse=None,
                    workspace: Optional[torch.Tensor] = None, stream=None):
    """O [B, Lq, Hq, d] bf16 and LSE [B, Hq, Lq] fp32 of the newest rows Q over the cache that holds their keys - the C entry
    point `seg_attn_decode`: row t of sequence b stands at slot kv_len - q_len + t and sees what seg_attn_fwd would show it
    (segments of S, tail T, one head class per KV head).  weights_out [B, Hkv, W] fp32, W >= max_pages * page_size, takes
    every slot's attention weight summed over the rows and query heads of its KV head, added to `weights` if given (which may
    be the same tensor).  Rows from q_len on, in O and in LSE, are left as they were."""
    c, B, Hkv, d, page, max_pages = _cache(K_pages, V_pages, block_table, kv_len, q_len, pos_shift, k_scale, v_scale)
    dev = K_pages.device
    if Q.dim() != 4 or Q.device != dev:
        raise ValueError("Q must be [B, Lq, Hq, d] on the cache's device")
    Lq, Hq = Q.shape[1], Q.shape[2]
    qs = _rows4(Q, (B, Lq, Hq, d), "Q")
    if out is None:
        out = torch.empty((B, Lq, Hq, d), dtype=torch.bfloat16, device=dev)
    elif out.device != dev:
        raise ValueError("out must be on the cache's device")
    os_ = _rows4(out, (B, Lq, Hq, d), "out")
    if lse is None:
        lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=dev)
    else:
        _flat(lse, torch.float32, (B, Hq, Lq), "lse", dev)
    W = 0
    if weights_out is not None:
        W = weights_out.shape[-1] if weights_out.dim() == 3 else 0
        _flat(weights_out, torch.float32, (B, Hkv, W), "weights_out", dev)
        _flat(weights, torch.float32, (B, Hkv, W), "weights", dev)
    elif weights is not None:
        raise ValueError("weights are added to in weights_out: pass that too (it may be the same tensor)")
    m = _mask_arr(head_past_mask, Hkv)
    L = lib()
    need = L.seg_attn_decode_workspace_bytes(c, Lq, Hq, int(weights_out is not None))
    ws = workspace
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    elif ws.device != dev:
        raise ValueError("workspace must be on the cache's device")
    _call(dev, L.seg_attn_decode, "seg_attn_decode", c, Lq, Hq, S, T, float(sm_scale if sm_scale is not None else d ** -0.5),
          m.ctypes.data, Q.data_ptr(), qs, out.data_ptr(), os_, lse.data_ptr(), _p(weights), _p(weights_out), W, ws.data_ptr(),
          ws.numel() * ws.element_size(), _on(dev, stream))
    return out, lse


def kv_evict(weights, K_pages, V_pages, block_table, kv_len, dst_table, sink: int, recent: int, heavy: int, pos_shift=None,
             k_scale=None, v_scale=None, weights_out=None, kv_len_out=None, pos_shift_out=None, workspace=None, stream=None):
    """Brings every sequence of more than sink + recent + heavy rows down to that many per KV head: the first `sink`, the last
    `recent` and the `heavy` rows of largest accumulated weight between them, copied in order to the pages of dst_table (int32
    [B, pages], none of them a page the sequence has now) - the C entry point `seg_kv_evict`.  weights is fp32 [B, Hkv, W] as
    seg_attn_decode gathers it.  Returns (idx int32 [B, Hkv, budget] (the slots kept, then -1), kv_len, pos_shift, weights) of
    the evicted cache, whose block table is dst_table; kv_len_out may be kv_len and pos_shift_out pos_shift."""
    c, B, Hkv, d, page, max_pages = _cache(K_pages, V_pages, block_table, kv_len, None, pos_shift, k_scale, v_scale)
    dev = K_pages.device
    if (dst_table.dim() != 2 or dst_table.dtype is not torch.int32 or dst_table.device != dev or dst_table.shape[0] != B or
            dst_table.stride(1) != 1 or (B > 1 and dst_table.stride(0) < dst_table.shape[1])):
        raise ValueError("dst_table must be an int32 tensor [B, pages] on %s with contiguous rows" % dev)
    W = weights.shape[-1] if weights.dim() == 3 else 0
    _flat(weights, torch.float32, (B, Hkv, W), "weights", dev)
    budget = sink + recent + heavy
    if min(sink, recent, heavy) < 0 or budget < 1:
        raise SegAttnError(1, "seg_kv_evict")
    idx = torch.empty((B, Hkv, budget), dtype=torch.int32, device=dev)
    weights_out = torch.empty((B, Hkv, W), dtype=torch.float32, device=dev) if weights_out is None else \
        _flat(weights_out, torch.float32, (B, Hkv, W), "weights_out", dev)
    kv_len_out = torch.empty((B,), dtype=torch.int32, device=dev) if kv_len_out is None else \
        _flat(kv_len_out, torch.int32, (B,), "kv_len_out", dev)
    pos_shift_out = torch.empty((B,), dtype=torch.int32, device=dev) if pos_shift_out is None else \
        _flat(pos_shift_out, torch.int32, (B,), "pos_shift_out", dev)
    L = lib()
    ws = workspace
    if ws is None:
        ws = torch.empty(max(L.seg_kv_evict_workspace_bytes(c), 256), dtype=torch.uint8, device=dev)
    elif ws.device != dev:
        raise ValueError("workspace must be on the cache's device")
    _call(dev, L.seg_kv_evict, "seg_kv_evict", c, weights.data_ptr(), W, sink, recent, heavy, dst_table.data_ptr(),
          dst_table.shape[1], dst_table.stride(0) if B > 1 else dst_table.shape[1], idx.data_ptr(), kv_len_out.data_ptr(),
          pos_shift_out.data_ptr(), weights_out.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _on(dev, stream))
    return idx, kv_len_out, pos_shift_out, weights_out
