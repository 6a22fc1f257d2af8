"""Serving from a paged key/value cache, and rotary positions in general form: the Python names of the C entry points
``seg_kv_append``, ``seg_attn_decode``, ``seg_kv_evict``, ``seg_rope_table_scaled`` and ``seg_rope_rotate``.

A cache is described by the same tensors in every call:

``K_pages``, ``V_pages``  ``[n_pages, page_size, Hkv, d]``, bf16 or ``torch.float8_e4m3fn``; any strides that are multiples
                          of 16 bytes with a contiguous last dimension (a permuted ``[n_pages, Hkv, page_size, d]`` buffer too)
``block_table``           int32 ``[B, max_pages]``: the pages of every sequence in order
``kv_len``                int32 ``[B]``: rows of every sequence, the call's new ones included
``q_len``                 int32 ``[B]`` or None: how many of the ``Lq`` rows given are there (the first ones); None: all
``pos_shift``             int32 ``[B]`` or None: rows that evictions have taken out (global position = slot + shift)
``k_scale``, ``v_scale``  fp32 ``[Hkv]``, for an 8-bit cache only (where its values are read or written)

Lengths stay on the device, so that a decoding step can be captured in a CUDA graph and replayed as they grow.
"""
from __future__ import annotations

import functools
import struct
from typing import Optional

import torch

from .binding import SegAttnError, _mask_arr, lib

_CACHE = struct.Struct("8i2P6q6P")     # seg_kv_cache
_STRIDE3 = struct.Struct("3q")
_SCALING = struct.Struct("i4x6d")      # seg_rope_scaling
_LAYOUTS = {"half": 0, "interleaved": 1}
_KINDS = {"plain": 0, "linear": 1, "by_parts": 2}
_BF16, _E4M3, _I32, _F32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32, torch.float32
# A decoding step's calls last a few microseconds on the device, so their way there counts: devices are compared by number,
# structures packed in one go, and the current stream and device are asked for as torch's own generated code asks for them (a
# Stream object costs as much as a launch).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _check(status: int, where: str):
    if status != 0:
        raise SegAttnError(status, where)


def _p(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _layout(name) -> int:
    if name not in _LAYOUTS:
        raise ValueError("layout must be 'half' or 'interleaved'")
    return _LAYOUTS[name]


def _rows4(t: torch.Tensor, shape, what: str, dev: int) -> bytes:
    """The (batch, row, head) strides of a bf16 tensor of this shape on CUDA device `dev`, the last dimension contiguous."""
    if t.dtype is not _BF16 or dev < 0 or t.get_device() != dev or t.shape != shape:
        raise ValueError("%s must be a bf16 CUDA tensor of shape %s on the device of the others" % (what, tuple(shape)))
    s = t.stride()
    if s[3] != 1:
        raise ValueError("%s must have a contiguous last dimension" % what)
    return _STRIDE3.pack(s[0], s[1], s[2])


def _flat(t, dtype, shape, what: str, dev: int):
    """A contiguous tensor of this type and shape on CUDA device `dev`."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on CUDA device %d" % (what, dtype, tuple(shape), dev))
    return t


def _call(dev: int, stream, fn, where: str, *args):
    """One C call with the tensors' device current, on the given stream of that device or its current one."""
    if stream is None:
        stream = _raw_stream(dev)
    elif stream.device_index != dev:
        raise ValueError("the stream belongs to another device than the tensors")
    else:
        stream = stream.cuda_stream
    if _current_device() == dev:
        _check(fn(*args, stream), where)
    else:
        with torch.cuda.device(dev):
            _check(fn(*args, stream), where)


def _on_stream(f):
    """`stream=`: the call runs with that stream current, so that what it allocates (results, workspaces) comes from the
    stream's own memory and is not handed to others while the kernels run."""
    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        if stream is None:
            return f(*args, **kw)
        with torch.cuda.stream(stream):
            return f(*args, stream=stream, **kw)
    return call


def _mask_bytes(head_past_mask, Hkv: int) -> bytes:
    """One head class per KV head, as seg_attn_fwd takes them."""
    if type(head_past_mask) in (list, tuple) and len(head_past_mask) == Hkv:
        try:
            return bytes(head_past_mask)
        except (TypeError, ValueError):
            pass
    return _mask_arr(head_past_mask, Hkv).tobytes()


def _cache(K, V, block_table, kv_len, q_len, pos_shift, k_scale, v_scale, reads_values: bool = True):
    """seg_kv_cache of these tensors as bytes, and (B, Hkv, d, page_size, max_pages, CUDA device)."""
    dev, kind = K.get_device(), K.dtype
    shape = K.shape
    if dev < 0 or len(shape) != 4 or shape != V.shape or V.get_device() != dev or V.dtype is not kind:
        raise ValueError("K_pages and V_pages must be CUDA tensors [n_pages, page_size, Hkv, d] of one shape, type and device")
    n_pages, page, Hkv, d = shape
    ks_ptr = vs_ptr = 0
    if kind is _E4M3:
        if reads_values:
            if k_scale is None or v_scale is None:
                raise ValueError("an 8-bit cache needs k_scale and v_scale")
            ks_ptr = _flat(k_scale, _F32, (Hkv,), "k_scale", dev).data_ptr()
            vs_ptr = _flat(v_scale, _F32, (Hkv,), "v_scale", dev).data_ptr()
    elif kind is not _BF16:
        raise ValueError("the cache must be bf16 or float8_e4m3fn")
    elif k_scale is not None or v_scale is not None:
        raise ValueError("scales belong to an 8-bit cache")
    k, v = K.stride(), V.stride()
    if k[3] != 1 or v[3] != 1:
        raise ValueError("the pages must have a contiguous last dimension")
    table = _pages(block_table, None, "block_table", dev)
    B = table[0]
    _flat(kv_len, _I32, (B,), "kv_len", dev)
    if q_len is not None:
        _flat(q_len, _I32, (B,), "q_len", dev)
    if pos_shift is not None:
        _flat(pos_shift, _I32, (B,), "pos_shift", dev)
    c = _CACHE.pack(B, Hkv, d, kind is _E4M3, page, n_pages, table[1], table[2], K.data_ptr(), V.data_ptr(), k[0], k[1], k[2], v[0],
                    v[1], v[2], ks_ptr, vs_ptr, block_table.data_ptr(), kv_len.data_ptr(), _p(q_len) or 0, _p(pos_shift) or 0)
    return c, B, Hkv, d, page, table[1], dev


def _pages(t, B, what: str, dev: int):
    """(B, entries of a row, elements between rows) of a table of page numbers."""
    if t.dtype is not _I32 or t.get_device() != dev or t.dim() != 2 or (B is not None and t.shape[0] != B):
        raise ValueError("%s must be an int32 tensor [B, pages] on CUDA device %d" % (what, dev))
    rows, n = t.shape
    s = t.stride()
    if (n > 1 and s[1] != 1) or (rows > 1 and s[0] < n):
        raise ValueError("%s must have contiguous rows that do not overlap" % what)
    return rows, n, s[0] if rows > 1 else n


@_on_stream
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
    table = torch.empty((n_pos, rot_dim // 2, 2), dtype=_F32, device=device)
    if not table.is_cuda:
        raise ValueError("the table lies on a CUDA device")
    sc = _SCALING.pack(_KINDS[kind], base, factor, trained_len, turns_lo, turns_hi, amplitude)
    _call(table.get_device(), stream, lib().seg_rope_table_scaled, "seg_rope_table_scaled", n_pos, rot_dim, sc, table.data_ptr())
    return table


def _table(table, dev: int):
    if table.dim() != 3 or table.shape[2] != 2 or table.dtype is not _F32 or table.get_device() != dev or not table.is_contiguous():
        raise ValueError("table must be a contiguous fp32 tensor [n_pos, rot_dim/2, 2] on CUDA device %d" % dev)
    return table.shape[0], 2 * table.shape[1]


@_on_stream
def rope_rotate(X, table, positions: Optional[torch.Tensor] = None, pos0: int = 0, layout: str = "half", inverse: bool = False,
                out: Optional[torch.Tensor] = None, stream=None):
    """Rows of X [B, L, H, d] rotated at `positions` (int32 [B, L]; None: pos0, pos0 + 1, ...) by a table of rope_table or
    rope_table_scaled, whose width is the part of the head that turns - the C entry point `seg_rope_rotate`.  `layout` names
    the pairs: "half" (x[i], x[i + rot/2]) or "interleaved" (x[2i], x[2i+1]).  inverse=True applies the transposed map, which
    takes the gradient of the output to that of X.  `out` may be X."""
    shape, dev = X.shape, X.get_device()
    if len(shape) != 4:
        raise ValueError("X must be [B, L, H, d]")
    xs = _rows4(X, shape, "X", dev)
    if out is None:
        out = torch.empty_like(X)
        ys = _STRIDE3.pack(*out.stride()[:3])
    else:
        ys = _rows4(out, shape, "out", dev)
    x, y = X.data_ptr(), out.data_ptr()
    if x == y and x and xs != ys:
        raise ValueError("a rotation in place needs the strides of X")
    n_pos, rot = _table(table, dev)
    B, L, H, d = shape
    if positions is not None:
        _flat(positions, _I32, (B, L), "positions", dev)
    _call(dev, stream, lib().seg_rope_rotate, "seg_rope_rotate", B, L, H, d, rot, _layout(layout), x, xs, y, ys, _p(positions), pos0,
          1 if inverse else 0, table.data_ptr(), n_pos)
    return out


@_on_stream
def kv_append(K_new, V_new, K_pages, V_pages, block_table, kv_len, table: Optional[torch.Tensor] = None, layout: str = "half",
              Q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, q_len=None, pos_shift=None, k_scale=None,
              v_scale=None, stream=None):
    """New rows K_new, V_new [B, Lq, Hkv, d] into the cache; with a table the keys, and the queries Q [B, Lq, Hq, d] if given,
    are rotated at their positions - the C entry point `seg_kv_append`.  Returns the rotated queries (q_out, which may be Q),
    or None.  kv_len counts the new rows already."""
    c, B, Hkv, d, _, _, dev = _cache(K_pages, V_pages, block_table, kv_len, q_len, pos_shift, k_scale, v_scale)
    if K_new.dim() != 4:
        raise ValueError("K_new and V_new must be [B, Lq, Hkv, d]")
    Lq = K_new.shape[1]
    kn, vn = _rows4(K_new, (B, Lq, Hkv, d), "K_new", dev), _rows4(V_new, (B, Lq, Hkv, d), "V_new", dev)
    n_pos = rot = Hq = 0
    if table is not None:
        n_pos, rot = _table(table, dev)
    qs = qo = None
    if Q is not None:
        if table is None:
            raise ValueError("queries are rotated by a table")
        Hq = Q.shape[2] if Q.dim() == 4 else 0
        qs = _rows4(Q, (B, Lq, Hq, d), "Q", dev)
        if q_out is None:
            q_out = torch.empty_like(Q)
        qo = _rows4(q_out, (B, Lq, Hq, d), "q_out", dev)
        if q_out.data_ptr() == Q.data_ptr() and qs != qo and Q.numel():
            raise ValueError("a rotation in place needs the strides of Q")
    elif q_out is not None:
        raise ValueError("q_out needs Q")
    _call(dev, stream, lib().seg_kv_append, "seg_kv_append", c, Lq, K_new.data_ptr(), kn, V_new.data_ptr(), vn, Hq, _p(Q), qs,
          _p(q_out), qo, _p(table), n_pos, rot, _layout(layout))
    return q_out


@_on_stream
def seg_attn_decode(Q, K_pages, V_pages, block_table, kv_len, S: int, T: int, head_past_mask=None, sm_scale: Optional[float] = None,
                    q_len=None, pos_shift=None, k_scale=None, v_scale=None, weights=None, weights_out=None, out=None, lse=None,
                    workspace: Optional[torch.Tensor] = None, stream=None):
    """O [B, Lq, Hq, d] bf16 and LSE [B, Hq, Lq] fp32 of the newest rows Q over the cache that holds their keys - the C entry
    point `seg_attn_decode`: row t of sequence b stands at slot kv_len - q_len + t and sees what seg_attn_fwd would show it
    (segments of S, tail T, one head class per KV head).  weights_out [B, Hkv, W] fp32, W >= max_pages * page_size, takes
    every slot's attention weight summed over the rows and query heads of its KV head, added to `weights` if given (which may
    be the same tensor).  Rows from q_len on, in O and in LSE, are left as they were.
    `out` may be Q, except with weights_out and more than 32 rows to a KV head (Hq/Hkv * Lq) of a bf16 cache."""
    c, B, Hkv, d, _, _, dev = _cache(K_pages, V_pages, block_table, kv_len, q_len, pos_shift, k_scale, v_scale)
    if Q.dim() != 4:
        raise ValueError("Q must be [B, Lq, Hq, d]")
    Lq, Hq = Q.shape[1], Q.shape[2]
    shape = (B, Lq, Hq, d)
    qs = _rows4(Q, shape, "Q", dev)
    if out is None:
        out = torch.empty_like(Q)
    os_ = _rows4(out, shape, "out", dev)
    if lse is None:
        lse = Q.new_empty((B, Hq, Lq), dtype=_F32)
    else:
        _flat(lse, _F32, (B, Hq, Lq), "lse", dev)
    W = 0
    if weights_out is not None:
        W = weights_out.shape[-1] if weights_out.dim() == 3 else 0
        _flat(weights_out, _F32, (B, Hkv, W), "weights_out", dev)
        if weights is not None:
            _flat(weights, _F32, (B, Hkv, W), "weights", dev)
    elif weights is not None:
        raise ValueError("weights are added to in weights_out: pass that too (it may be the same tensor)")
    L = lib()
    if workspace is None:
        need = L.seg_attn_decode_workspace_bytes(c, Lq, Hq, 0 if weights_out is None else 1)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=Q.device)
    elif workspace.get_device() != dev:
        raise ValueError("workspace must be on the cache's device")
    _call(dev, stream, L.seg_attn_decode, "seg_attn_decode", c, Lq, Hq, S, T, d ** -0.5 if sm_scale is None else sm_scale,
          _mask_bytes(head_past_mask, Hkv), Q.data_ptr(), qs, out.data_ptr(), os_, lse.data_ptr(), _p(weights), _p(weights_out), W,
          workspace.data_ptr(), workspace.nbytes)
    return out, lse


@_on_stream
def kv_evict(weights, K_pages, V_pages, block_table, kv_len, dst_table, sink: int, recent: int, heavy: int, pos_shift=None,
             weights_out=None, kv_len_out=None, pos_shift_out=None, stream=None):
    """Brings every sequence of more than sink + recent + heavy rows down to that many per KV head: the first `sink`, the last
    `recent` and the `heavy` rows of largest accumulated weight between them, copied in order to the pages of dst_table (int32
    [B, pages], none of them a page the sequence has now) - the C entry point `seg_kv_evict`.  Rows are moved as they are: an
    8-bit cache's scales are not needed.  weights is fp32 [B, Hkv, W] as
    seg_attn_decode gathers it.  Returns (idx int32 [B, Hkv, budget] (the slots kept, then -1), kv_len, pos_shift, weights) of
    the evicted cache, whose block table is dst_table; kv_len_out may be kv_len and pos_shift_out pos_shift."""
    c, B, Hkv, d, _, _, dev = _cache(K_pages, V_pages, block_table, kv_len, None, pos_shift, None, None, reads_values=False)
    _, dst_pages, dst_stride = _pages(dst_table, B, "dst_table", dev)
    W = weights.shape[-1] if weights.dim() == 3 else 0
    _flat(weights, _F32, (B, Hkv, W), "weights", dev)
    budget = sink + recent + heavy
    if min(sink, recent, heavy) < 0 or budget < 1:
        raise SegAttnError(1, "seg_kv_evict")
    idx = kv_len.new_empty((B, Hkv, budget))
    weights_out = torch.empty_like(weights) if weights_out is None else _flat(weights_out, _F32, (B, Hkv, W), "weights_out", dev)
    kv_len_out = torch.empty_like(kv_len) if kv_len_out is None else _flat(kv_len_out, _I32, (B,), "kv_len_out", dev)
    pos_shift_out = torch.empty_like(kv_len) if pos_shift_out is None else _flat(pos_shift_out, _I32, (B,), "pos_shift_out", dev)
    _call(dev, stream, lib().seg_kv_evict, "seg_kv_evict", c, weights.data_ptr(), W, sink, recent, heavy, dst_table.data_ptr(), dst_pages,
          dst_stride, idx.data_ptr(), kv_len_out.data_ptr(), pos_shift_out.data_ptr(), weights_out.data_ptr())
    return idx, kv_len_out, pos_shift_out, weights_out
