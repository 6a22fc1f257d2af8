"""Pages from requested lengths, blocks with scales, their means and their choice, and the attention over them: from their definitions,
one sequence at a time, in whole numbers and 64 bits."""
import math

import numpy as np
import torch

import paged_ref as ref

E4M3 = torch.float8_e4m3fn
bits = lambda t: t.view(torch.uint8) if t.dtype == E4M3 else t.view(torch.int16)  # noqa: E731


def resize(want, table, lens, free, count, page, Lq, shift=None, cap=None):
    """Lists of Python integers in, (table, kv_len, free list, q_len, slots, positions) out; every number in range."""
    table, free = [list(r) for r in table], list(free[:count])
    cap = len(table[0]) * page if cap is None else cap
    pages = lambda n: -(-n // page)
    want = [w if 0 <= w <= cap and w - n <= Lq else n for w, n in zip(want, lens)]
    for b, (w, n) in enumerate(zip(want, lens)):
        free += table[b][pages(w):pages(n)]
    out, full = list(lens), False
    for b, (w, n) in enumerate(zip(want, lens)):
        need = pages(w) - pages(n)
        if need > 0:
            full = full or need > len(free)
            if full:
                continue
            for k in range(pages(n), pages(w)):
                table[b][k] = free.pop()
        out[b] = w
    q = [max(0, o - n) for o, n in zip(out, lens)]
    slots, pos = [[-1] * Lq for _ in lens], [[0] * Lq for _ in lens]
    for b, n in enumerate(lens):
        for t in range(q[b]):
            s = n + t
            slots[b][t], pos[b][t] = table[b][s // page] * page + s % page, s + (shift[b] if shift else 0)
    return table, out, free, q, slots, pos


def scale_of(top):
    """The smallest power of two that brings `top` within 448, as a float; from 2^-40 to 2^119."""
    if top <= 0:
        return 2.0 ** -40
    m, e = math.frexp(float(top))
    return 2.0 ** min(max(e - 9 + (1 if m > 0.875 else 0), -40), 119)


def append(pages, scales, rows, new, first, n, table, page):
    """Rows `new` (float32 [n - first, Hkv, d]) to slots first..n-1 of one sequence, in place: 8-bit pages and scales on the CPU."""
    slot = first
    while slot < n:
        start = slot // rows * rows
        end = min(n, start + rows)
        at, row = table[start // page], start % page
        x = new[slot - first:end - first]
        for h in range(x.shape[1]):
            a = x[:, h].abs()
            top = a[torch.isfinite(a)].max().item() if torch.isfinite(a).any() else 0.0
            s, old = scale_of(top), scales[at, row // rows, h].item()
            if start < slot:
                if s > old:
                    was = pages[at, row:row + slot - start, h].float() * torch.tensor(old / s)
                    bits(pages)[at, row:row + slot - start, h] = bits(was.clamp(-448, 448).to(E4M3))
                else:
                    s = old
            scales[at, row // rows, h] = s
            y = (x[:, h] * (1 / torch.tensor(s))).clamp(-448, 448).to(E4M3)
            bits(pages)[at, row + slot - start:row + end - start, h] = bits(y)
        slot = end


def dequantised(pages, scale, rows=None):
    """Pages as float64 [n_pages, page, Hkv, d]; scale: None, [Hkv], or [n_pages, page / rows, Hkv]."""
    x = pages.float().cpu().double().numpy()
    if scale is None:
        return x
    s = scale.cpu().double().numpy()
    return x * (s[:, None] if s.ndim == 1 else np.repeat(s, x.shape[1] // s.shape[1], 1)[..., None])


def by_row(scale, page, n_pages=0):
    """Scales [Hkv] or [n_pages, page / rows, Hkv] as float64 [n_pages, page, Hkv]; n_pages is given for the first."""
    s = scale.cpu().double().numpy()
    return np.broadcast_to(s, (n_pages, page, len(s))) if s.ndim == 1 else np.repeat(s, page // s.shape[1], 1)


def means(x, block):
    """x: float64 [rows, Hkv, d] of one full block -> (int8 [Hkv, d], fp32 [Hkv])."""
    with np.errstate(all="ignore"):
        m = (x.sum(0) / block).astype(np.float32)
        top = np.abs(m).max(-1)
        fine = np.isfinite(m).all(-1)
        scale = np.where(fine, top * (np.float32(1) / np.float32(127)), np.float32(np.nan)).astype(np.float32)
        q = np.where((fine & (scale > 0))[:, None], np.rint(m / scale[:, None]), 0)
    return np.nan_to_num(q, nan=0.0).astype(np.int8), scale


def first_whole(pos, S, T, shift, block):
    return ref.lowest_visible(pos, S, T, ref.LOCAL, shift) // block * block


def select(Q, sums, scale, table, n, q_len, S, T, mask, page, block, count, sink, shift=0):
    """Q float64 [q_len, Hq, d] of one sequence; sums, scale: numpy.  -> int [q_len, Hkv, count]."""
    Hkv, per = sums.shape[2], page // block
    g = Q.shape[1] // Hkv
    out = np.full((q_len, Hkv, count), -1, np.int64)
    for t in range(q_len):
        slot = n - q_len + t
        if slot < 0:
            continue
        room = first_whole(slot + shift, S, T, shift, block) // block
        for h in range(Hkv):
            if mask[h] != ref.PAST or room == 0:
                continue
            s = Q[t, h * g:(h + 1) * g].sum(0).astype(np.float32)
            top = np.abs(s).max()
            step = top * (np.float32(1) / np.float32(127))
            p = np.rint(s / step).astype(np.int64) if np.isfinite(top) and step > 0 else np.zeros(len(s), np.int64)
            j = np.arange(room)
            pg = np.asarray(table)[j * block // page]
            k, c = sums[pg, j % per, h].astype(np.int64), scale[pg, j % per, h]
            with np.errstate(invalid="ignore"):
                score = (k @ p).astype(np.float32) * c
            rank = sorted(range(room), key=lambda i: (i >= sink, math.isnan(score[i]), -score[i] if not math.isnan(score[i]) else 0.0, i))
            out[t, h, :min(room, count)] = sorted(rank[:count])
    return out


def visible(n, q_len, t, cls, S, T, shift, chosen=None, block=0):
    """Slots that new row t of a sequence sees; chosen: its list of blocks, or None."""
    e = n - q_len + t
    if e < 0:
        return np.arange(0)
    if chosen is None or cls != ref.PAST:
        return np.arange(ref.lowest_visible(e + shift, S, T, cls, shift), e + 1)
    low = first_whole(e + shift, S, T, shift, block)
    far = []
    for k in chosen:
        if not 0 <= k < low // block or (far and k <= far[-1]):
            break
        far.append(int(k))
    return np.concatenate([np.arange(k * block, (k + 1) * block) for k in far] + [np.arange(low, e + 1)]).astype(int)


def attend(Q, K, V, table, lens, q_len, S, T, mask, scale, page, shift=None, idx=None, block=0, cap=0, v_scale=None):
    """paged_ref.decode with chosen blocks and values of any scale: K, V float64 [n_pages, page, Hkv, d].  v_scale: the scales of an 8-bit
    V by row, [n_pages, page, Hkv].  Its weights times their scales are fp16 numbers, the largest of them 2^12 at least, and those under
    fp16's normal range are off by up to half a step of it, 2^-25, whatever they are: 2^-37 of the largest weight times scale, for each
    stored value.  That is added to `spread`, which check_decode multiplies by 2^-11."""
    B, Lq, Hq, d = Q.shape
    Hkv = K.shape[2]
    g = Hq // Hkv
    O, lse = np.full((B, Lq, Hq, d), np.nan), np.full((B, Hq, Lq), np.nan)
    spread, terms, w = np.zeros((B, Lq, Hq, d)), np.zeros((B, Hq, Lq)), np.zeros((B, Hkv, cap))
    for b in range(B):
        sh = 0 if shift is None else int(shift[b])
        for t in range(q_len[b]):
            for h in range(Hkv):
                j = visible(lens[b], q_len[b], t, mask[h], S, T, sh, None if idx is None else idx[b, t, h], block)
                at = np.asarray(table[b])[j // page], j % page, h
                for q in range(h * g, (h + 1) * g):
                    if not len(j):
                        O[b, t, q], lse[b, q, t] = 0.0, -np.inf
                        continue
                    s = scale * (K[at] @ Q[b, t, q])
                    m = s.max()
                    p = np.exp(s - m)
                    z = p.sum()
                    p /= z
                    O[b, t, q], spread[b, t, q] = p @ V[at], p @ np.abs(V[at])
                    if v_scale is not None:
                        vs = v_scale[at]
                        spread[b, t, q] += 2.0 ** -37 / ref.FP16 * (p * vs).max() * np.abs(V[at] / vs[:, None]).sum(0)
                    lse[b, q, t] = m + math.log(z)
                    terms[b, q, t] = scale * (np.abs(K[at]) @ np.abs(Q[b, t, q])).max()
                    if cap:
                        w[b, h, j] += p
    return O, lse, spread, terms, w


class ScaledCache(ref.Cache):
    """A cache in 8 bits whose blocks have scales of their own, of any value (`powers`: powers of two, as an append leaves them); scales
    of blocks that nobody owns are NaN."""

    def __init__(self, lens, Hkv, d, page, rows, seed=0, powers=True, spread=3, **kw):
        super().__init__(lens, Hkv, d, page, fp8=True, seed=seed, **kw)
        g = torch.Generator().manual_seed(100 + seed)
        shape = (self.K.shape[0], page // rows, Hkv)
        self.rows, owned = rows, torch.zeros(shape[:2], dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(0, n, rows):
                owned[self.table[b, j // page].long(), j % page // rows] = True
        out = []
        for _ in range(2):
            s = torch.exp2(torch.randint(-spread, spread + 1, shape, generator=g).float() - 2)
            if not powers:
                s = s * (1 + torch.rand(shape, generator=g))
            s[~owned] = math.nan
            out.append(s)
        self.k_scale, self.v_scale = out
        # strides of their own: [n_pages, Hkv, blocks] underneath
        to = lambda s: s.transpose(1, 2).contiguous().to(self.K.device).transpose(1, 2)
        self.scales = dict(k_scale=to(out[0]), v_scale=to(out[1]))

    def values(self):
        return dequantised(self.K, self.scales["k_scale"]), dequantised(self.V, self.scales["v_scale"])
