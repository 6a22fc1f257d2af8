"""The paged-cache operators and the rotary forms in 64 bits, written from their definitions, one row at a time."""
import math

import numpy as np
import torch

LOCAL, PAST, OWN = 0, 1, 2
BF16, FP16, FP32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24     # half a step, relative to the value
NAN8 = 0x7f


def frequencies(rot, base=10000.0, kind="plain", factor=1.0, trained_len=0.0, turns_lo=0.0, turns_hi=0.0):
    w = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if kind == "linear":
        w = [x / factor for x in w]
    if kind == "by_parts":
        out = []
        for x in w:
            turns = trained_len * x / (2 * math.pi)
            g = min(max((turns - turns_lo) / (turns_hi - turns_lo), 0.0), 1.0)
            out.append((1 - g) * x / factor + g * x)
        w = out
    return np.array(w)


def pairs(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(x, table, layout, inverse=False):
    """Rows x [..., H, d] turned by table rows [..., rot/2, 2], in the type of x (float32: operation by operation)."""
    rot = 2 * table.shape[-2]
    a, b = pairs(rot, layout)
    c, s = table[..., None, :, 0].astype(x.dtype), table[..., None, :, 1].astype(x.dtype)
    s = -s if inverse else s
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def lowest_visible(pos, S, T, cls, shift):
    start = pos // S * S
    if cls == PAST:
        return 0
    return max(0, (max(0, start - T) if cls == LOCAL else start) - shift)


def rows_of(pages, table_row, n, page):
    """Rows 0..n-1 of a sequence as float64 [n, Hkv, d]."""
    j = np.arange(n)
    x = pages.float().cpu().double().numpy() if torch.is_tensor(pages) else pages
    return x[np.asarray(table_row)[j // page], j % page]


def decode(Q, K, V, table, kv_len, q_len, S, T, mask, scale, page, shift=None, k_scale=None, v_scale=None, bad_pages=()):
    """Per row: O, LSE, and what a bound needs: sum of p|v|, the largest score's term sum; and the summed weights
    [B, Hkv, cap].  Rows that are not there come out as NaN."""
    B, Lq, Hq, d = Q.shape
    Hkv = K.shape[2]
    g = Hq // Hkv
    cap = table.shape[1] * page
    O = np.full((B, Lq, Hq, d), np.nan)
    lse = np.full((B, Hq, Lq), np.nan)
    spread = np.zeros((B, Lq, Hq, d))
    terms = np.zeros((B, Hq, Lq))
    w = np.zeros((B, Hkv, cap))
    for b in range(B):
        n = int(kv_len[b])
        sh = 0 if shift is None else int(shift[b])
        tb = np.where(table[b] < 0, 0, table[b])
        Kb, Vb = rows_of(K, tb, n, page), rows_of(V, tb, n, page)
        if k_scale is not None:
            Kb, Vb = Kb * k_scale[:, None], Vb * v_scale[:, None]
        for t in range(int(q_len[b])):
            e = n - int(q_len[b]) + t
            for h in range(Hkv):
                j = np.arange(lowest_visible(e + sh, S, T, mask[h], sh), e + 1) if e >= 0 else np.arange(0)
                j = np.array([x for x in j if table[b][x // page] not in bad_pages], dtype=int) if len(bad_pages) else j
                for q in range(h * g, (h + 1) * g):
                    if not len(j):
                        O[b, t, q], lse[b, q, t] = 0.0, -np.inf
                        continue
                    s = scale * (Kb[j, h] @ Q[b, t, q])
                    m = s.max()
                    p = np.exp(s - m)
                    z = p.sum()
                    p /= z
                    O[b, t, q] = p @ Vb[j, h]
                    spread[b, t, q] = p @ np.abs(Vb[j, h])
                    lse[b, q, t] = m + math.log(z)
                    terms[b, q, t] = scale * (np.abs(Kb[j, h]) @ np.abs(Q[b, t, q])).max()
                    w[b, h, j] += p
    return O, lse, spread, terms, w


def check_decode(O, lse, ref, Lq_rows, d, fp8=False, w_in=None, w_out=None, kv_len=None):
    """Against decode()'s answer.  With u = 2^-24: a score is a sum of d products in fp32 and two scalings, off by at most
    (d + 3) u times the sum of its terms' magnitudes; exp2 and the running rescalings add a few u each, and a sum over n keys
    split and joined at most n u, here n <= 2^14 in the worst order (2^-10, met by no tree: pairwise order gives 20 u, and
    what is allowed is 2^-18).  A weight is then off by its score's and the normaliser's error, relatively; the weights are
    rounded to 16 bits before the product (2^-8 for bf16, 2^-11 for fp16), the output once to bf16."""
    Or, lr, spread, terms, w = ref
    es = (d + 8) * FP32 * terms + 2.0 ** -18
    there = np.isfinite(lr)
    O, lse = O.float().cpu().double().numpy(), lse.cpu().double().numpy()
    for b, rows in enumerate(Lq_rows):
        for t in range(rows):
            assert np.array_equal(np.isfinite(lse[b, :, t]), there[b, :, t]), (b, t)
            fin = there[b, :, t]
            assert (lse[b, ~fin, t] == -np.inf).all() and (O[b, t, ~fin] == 0).all()
            err = np.abs(lse[b, fin, t] - lr[b, fin, t])
            assert (err <= es[b, fin, t] + 4 * FP32 * np.abs(lr[b, fin, t])).all(), ("lse", b, t, float(err.max()))
            bound = ((FP16 if fp8 else BF16) + 2 * es[b, :, t, None]) * spread[b, t] + BF16 * 1.02 * np.abs(Or[b, t]) + 1e-30
            err = np.abs(O[b, t] - Or[b, t])
            assert (err <= bound).all(), ("O", b, t, float((err / bound).max()))
    if w_out is not None:
        got = w_out.cpu().double().numpy()
        base = np.zeros_like(w) if w_in is None else w_in.cpu().double().numpy()[..., :w.shape[-1]]
        for b, rows in enumerate(Lq_rows):
            if rows == 0:
                continue
            n = int(kv_len[b])
            want = base[b, :, :n] + w[b, :, :n]
            bound = 2 * es[b].max() * w[b, :, :n] + 2 * FP32 * np.abs(want) + 1e-37
            err = np.abs(got[b, :, :n] - want)
            assert (err <= bound).all(), ("weights", b, float((err / bound).max()))


def evict_choice(w, n, sink, recent, heavy):
    """The slots one KV head keeps, ascending."""
    if n <= sink + recent + heavy:
        return list(range(n))
    mid = [(0, 0.0, -j) if math.isnan(float(w[j])) else (1, float(w[j]), -j) for j in range(sink, n - recent)]
    best = sorted(mid, reverse=True)[:heavy]
    return sorted(list(range(sink)) + [-x[2] for x in best] + list(range(n - recent, n)))


class Cache:
    """A paged cache with shuffled pages; the rows of pages nobody owns, and rows behind a sequence's end, are NaN."""

    def __init__(self, lens, Hkv, d, page, fp8=False, seed=0, max_pages=None, head_major=False, spare=3, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.page, self.lens = page, list(lens)
        need = [-(-n // page) for n in lens]
        self.max_pages = max(1, max(need, default=1)) if max_pages is None else max_pages
        B, n_pages = len(lens), sum(need) + spare
        order = torch.randperm(n_pages, generator=g)
        self.table = torch.full((B, self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        self.spare = order[at:].tolist()
        shape = (n_pages, Hkv, page, d) if head_major else (n_pages, page, Hkv, d)
        k, v = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
        if head_major:
            k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                used[self.table[b, j // page].long(), j % page] = True
        k[~used], v[~used] = math.nan, math.nan
        self.k_scale = self.v_scale = None
        if fp8:
            self.k_scale, self.v_scale = torch.rand(Hkv, generator=g) + 0.05, torch.rand(Hkv, generator=g) + 0.05
            k, v = 4 * k, 4 * v
        kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
        self.K, self.V = k.to(kind).to(device), v.to(kind).to(device)
        if head_major:   # .to() keeps the strides of a dense permuted tensor
            assert self.K.stride(1) == d and self.K.stride(2) == page * d
        self.dev = dict(block_table=self.table.to(device), kv_len=torch.tensor(lens, dtype=torch.int32, device=device))
        self.scales = {} if not fp8 else dict(k_scale=self.k_scale.to(device), v_scale=self.v_scale.to(device))

    def ref_scales(self):
        return {} if self.k_scale is None else dict(k_scale=self.k_scale.double().numpy(), v_scale=self.v_scale.double().numpy())
