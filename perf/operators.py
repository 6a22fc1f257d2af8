"""The operators of serving from a paged key/value cache: what is measured, and their plain forms.

Four operators share one description of the cache: K and V pages [n_pages, page_size, Hkv, d] (bf16, or e4m3 with one
scale per KV head), a block table [B, max_pages] of page numbers, and the length of every sequence.

  decode   attention of each sequence's newest tokens over its cache, under the segment mask of the head's class
  append   new keys and values into the cache, the keys (and the queries) rotated by their positions
  evict    the slots of largest accumulated attention weight, and what must stay, copied to other pages
  rope     the rotation alone, forward or transposed (its backward pass), in either pairing, on part of the head
"""
import math
import random

import numpy as np
import torch

own = False   # false: the plain forms below; true: the calls a user makes of the framework


def listed():
    return [
        # one user's short chat turn: a single new token over half a thousand slots; latency is all that counts
        dict(name="decode_one_short", op="decode", B=1, lo=517, hi=517, Lq=1, Hq=32, Hkv=8, d=128, S=2048, T=512, past=2, page=16,
             fp8=False, weights=False),
        # a full serving batch with prompts of every length, the head classes of the 16K configuration
        dict(name="decode_ragged", op="decode", B=64, lo=1, hi=16384, Lq=1, Hq=32, Hkv=8, d=128, S=2048, T=512, past=2, page=64,
             fp8=False, weights=False),
        # the 128K configuration served from an 8-bit cache
        dict(name="decode_128k_fp8", op="decode", B=8, lo=100000, hi=131072, Lq=1, Hq=32, Hkv=8, d=128, S=8192, T=2048, past=2,
             page=128, fp8=True, weights=False),
        # every head reads its whole past, eight query heads to a KV head: the largest read
        dict(name="decode_all_past", op="decode", B=16, lo=16384, hi=32768, Lq=1, Hq=64, Hkv=8, d=128, S=4096, T=1024, past=8, page=64,
             fp8=False, weights=False),
        # the last 16 tokens of a prompt as an observation window: their attention weights are summed for an eviction
        dict(name="decode_window_weights", op="decode", B=4, lo=12000, hi=16384, Lq=16, Hq=32, Hkv=8, d=128, S=4096, T=1024, past=4,
             page=64, fp8=False, weights=True),
        # one new token for each sequence of a serving batch
        dict(name="append_tokens", op="append", B=64, lo=100, hi=8000, Lq=1, Hq=32, Hkv=8, d=128, rot=128, pairs="half", page=16,
             fp8=False),
        # a prompt chunk of 8192 tokens for two sequences, neighbouring elements paired, half of the head rotated
        dict(name="append_chunk", op="append", B=2, lo=8192, hi=20000, Lq=8192, Hq=32, Hkv=8, d=128, rot=64, pairs="interleaved",
             page=64, fp8=False),
        # a prompt chunk into an 8-bit cache
        dict(name="append_chunk_fp8", op="append", B=3, lo=1500, hi=9001, Lq=4096, Hq=32, Hkv=8, d=128, rot=128, pairs="half", page=64,
             fp8=True),
        # one sequence outgrows a small budget
        dict(name="evict_one", op="evict", B=1, lo=4133, hi=4133, Hkv=8, d=128, sink=4, recent=640, heavy=380, page=16, fp8=False),
        # a batch of long sequences brought down to a third
        dict(name="evict_batch", op="evict", B=16, lo=20000, hi=32768, Hkv=8, d=128, sink=16, recent=5120, heavy=2900, page=64, fp8=False),
        # one token's query heads, half layout
        dict(name="rope_tokens", op="rope", B=8, L=1, H=32, d=128, rot=128, pairs="half", inverse=False),
        # the gradient of a 16K training batch's queries rotated back, neighbouring elements paired, three quarters of the head
        dict(name="rope_backward", op="rope", B=2, L=16384, H=32, d=128, rot=96, pairs="interleaved", inverse=True),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "append", "evict", "rope"])
    d, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8])
    page = rng.choice([8, 16, 48, 64, 100, 128, 256])
    fp8 = rng.random() < 0.4
    B = _log(rng, 1, 64)
    if op == "decode":
        hi = _log(rng, 1, min(131072, 400000 // B))
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        S = _log(rng, 64, 16384)
        return dict(op=op, B=B, lo=max(1, int(hi * rng.random())), hi=hi, Lq=rng.choice([1, 1, 1, 2, 5]), Hq=Hq, Hkv=Hkv, d=d, S=S,
                    T=rng.randint(0, S), past=rng.randint(0, Hkv), page=page, fp8=fp8, weights=rng.random() < 0.3)
    if op == "append":
        Lq = _log(rng, 1, 16384 // B)
        hi = Lq + _log(rng, 1, 4000)
        return dict(op=op, B=B, lo=Lq, hi=hi, Lq=Lq, Hq=Hkv * rng.choice([1, 2, 4]), Hkv=Hkv, d=d, rot=rng.choice([16, 32, 48, 64, d]),
                    pairs=rng.choice(["half", "interleaved"]), page=page, fp8=fp8)
    if op == "evict":
        hi = _log(rng, 300, min(131072, 500000 // B))
        recent, heavy = int(hi * rng.uniform(0.02, 0.3)), int(hi * rng.uniform(0.02, 0.3))
        return dict(op=op, B=B, lo=max(1, int(hi * rng.uniform(0.3, 1))), hi=hi, Hkv=Hkv, d=d, sink=rng.randint(0, 16), recent=recent,
                    heavy=heavy, page=page, fp8=fp8)
    return dict(op=op, B=B, L=_log(rng, 1, 32768 // B), H=rng.choice([1, 5, 8, 32]), d=d, rot=rng.choice([16, 32, 48, 64, d]),
                pairs=rng.choice(["half", "interleaved"]), inverse=rng.random() < 0.5)


def _lengths(c):
    """The sequences' lengths, and how many tokens of each are new (a case's own, whatever the seed)."""
    r = random.Random("%d %d %d" % (c["B"], c["lo"], c["hi"]))
    n = [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])]
    n[-1] = c["hi"]
    new = [min(x, c.get("Lq", 1)) for x in n]
    return n, new


def _classes(c):
    # `past` of the KV heads read everything older, spread over the heads; the others their segment and its carried tail
    return [int((h * c["past"]) // c["Hkv"] != ((h + 1) * c["past"]) // c["Hkv"]) for h in range(c["Hkv"])]


def _angles(n_pos, rot):
    # positions interpolated by parts for a context eight times the trained 16384: frequencies of under one turn over the
    # trained length are divided by 8, those of over 32 turns kept, a ramp between; cosines and sines in double
    w = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    g = ((16384.0 * w / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * ((1 - g) * w / 8.0 + g * w)
    return torch.stack([a.cos(), a.sin()], -1).float()


def prepare(case, seed):
    c, s = case, {}
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    s["case"] = c
    if c["op"] == "rope":
        s["X"] = normal(c["B"], c["L"], c["H"], c["d"])
        first = torch.randint(0, 1000, (c["B"], 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(c["L"], device="cuda")).int()
        s["table"] = _angles(c["L"] + 1000, c["rot"])
        return s
    B, Hkv, d, page = c["B"], c["Hkv"], c["d"], c["page"]
    n, new = _lengths(c)
    need = [-(-x // page) for x in n]
    per, total = max(need), sum(need)
    kept = c["sink"] + c["recent"] + c["heavy"] if c["op"] == "evict" else 0
    dst_per = -(-kept // page)
    pages = total + B * dst_per
    order = torch.randperm(pages, generator=g, device="cuda").int()   # pages are handed out in no order
    table = torch.full((B, per), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    s["block_table"] = table
    s["kv_len"] = torch.tensor(n, dtype=torch.int32, device="cuda")
    s["K"], s["V"] = normal(pages, page, Hkv, d), normal(pages, page, Hkv, d)
    s["k_scale"] = s["v_scale"] = None
    if c["fp8"]:
        s["K"], s["V"] = (16 * s["K"]).to(torch.float8_e4m3fn), (16 * s["V"]).to(torch.float8_e4m3fn)
        s["k_scale"], s["v_scale"] = ((0.5 + torch.rand(Hkv, generator=g, device="cuda")) / 16 for _ in range(2))
    if c["op"] == "evict":
        s["dst_table"] = order[at:].reshape(B, dst_per).contiguous()
        # accumulated weights: a few large, most small, and many slots that nothing ever looked at
        w = torch.rand((B, Hkv, per * page), generator=g, device="cuda")
        s["weights"] = w.pow(8) * (torch.rand(w.shape, generator=g, device="cuda") > 0.1)
        return s
    s["q_len"] = torch.tensor(new, dtype=torch.int32, device="cuda") if min(new) < c["Lq"] else None
    s["Q"] = normal(B, c["Lq"], c["Hq"], d)
    if c["op"] == "decode":
        s["mask"] = _classes(c)
        s["O"] = torch.zeros_like(s["Q"])
        s["LSE"] = torch.zeros((B, c["Hq"], c["Lq"]), device="cuda")
        if c["weights"]:
            s["weights"] = torch.rand((B, Hkv, per * page), generator=g, device="cuda")
            s["weights_out"] = torch.zeros_like(s["weights"])
    else:
        s["Kn"], s["Vn"] = normal(B, c["Lq"], Hkv, d), normal(B, c["Lq"], Hkv, d)
        s["Qr"] = torch.zeros_like(s["Q"])
        s["angles"] = _angles(max(n), c["rot"])
    return s


def run(s):
    return {"decode": _decode, "append": _append, "evict": _evict, "rope": _rope}[s["case"]["op"]](s)


# ---- plain forms, in 32 bits ----------------------------------------------------------------------------------------

def _new_slots(s):
    """Slot of every new row [B, Lq] and whether the row is there at all."""
    c, n = s["case"], s["kv_len"].long()
    t = torch.arange(c["Lq"], device="cuda")
    new = n.clamp(max=c["Lq"]) if s["q_len"] is None else s["q_len"].long()
    return (n - new)[:, None] + t, t < new[:, None]


def _bits(x):
    # 8-bit values are moved as bytes
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _rows(s, name, scale):
    """The cache's rows as 32-bit values [B, slots, Hkv, d] (slots behind a sequence's end: any row)."""
    c = s["case"]
    j = torch.arange(s["block_table"].shape[1] * c["page"], device="cuda")
    x = _bits(s[name])[s["block_table"].long().clamp(min=0)[:, j // c["page"]], (j % c["page"])[None]].view(s[name].dtype).float()
    return x if s[scale] is None else x * s[scale][:, None]


def _visible(s, slots):
    """[B, Hkv, Lq, slots]: what a row may see by its KV head's class; rows that are not there see nothing."""
    c = s["case"]
    p, there = _new_slots(s)
    start = p // c["S"] * c["S"]
    low = (start - c["T"]).clamp(min=0)[:, None] * (1 - torch.tensor(s["mask"], device="cuda"))[None, :, None]
    j = torch.arange(slots, device="cuda")
    return (j >= low[..., None]) & (j <= p[:, None, :, None]) & there[:, None, :, None]


def _decode(s):
    c = s["case"]
    B, Lq, Hq, Hkv, d = c["B"], c["Lq"], c["Hq"], c["Hkv"], c["d"]
    if own:
        import paper_2605_11744_b200 as sa
        more = dict(weights=s["weights"], weights_out=s["weights_out"]) if c["weights"] else {}
        sa.seg_attn_decode(s["Q"], s["K"], s["V"], s["block_table"], s["kv_len"], c["S"], c["T"], s["mask"], q_len=s["q_len"],
                           k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["O"], lse=s["LSE"], **more)
        return [s["O"], s["LSE"]] + ([s["weights_out"]] if c["weights"] else [])
    K = _rows(s, "K", "k_scale")
    q = s["Q"].float().reshape(B, Lq, Hkv, Hq // Hkv, d)
    x = torch.einsum("btcgd,bjcd->bcgtj", q, K) * d ** -0.5
    del K
    x = x.masked_fill(~_visible(s, x.shape[-1])[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = (x - m.masked_fill(m == -math.inf, 0.0)).exp()
    z = e.sum(-1, keepdim=True)
    P = e / z.masked_fill(z == 0, 1.0)
    lse = (m + z.log()).squeeze(-1).reshape(B, Hq, Lq)
    O = torch.einsum("bcgtj,bjcd->btcgd", P, _rows(s, "V", "v_scale")).reshape(B, Lq, Hq, d).bfloat16()
    there = _new_slots(s)[1]
    got = [torch.where(there[:, :, None, None], O, s["O"]), torch.where(there[:, None], lse, s["LSE"])]
    if c["weights"]:
        inside = torch.arange(x.shape[-1], device="cuda") < s["kv_len"][:, None]
        got.append(torch.where(inside[:, None], s["weights"] + P.sum((2, 3)), s["weights_out"]))
    return got


def _turn(x, cs, c, inverse=False):
    """x [B, L, H, d] in 32 bits rotated by cs [B, L, rot/2, 2]."""
    r = c["rot"]
    cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
    sin = -sin if inverse else sin
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["pairs"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([y, z], -1) if c["pairs"] == "half" else torch.stack([y, z], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _append(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        sa.kv_append(s["Kn"], s["Vn"], s["K"], s["V"], s["block_table"], s["kv_len"], table=s["angles"], layout=c["pairs"], Q=s["Q"],
                     q_out=s["Qr"], q_len=s["q_len"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return [s["K"], s["V"], s["Qr"]]
    slot, there = _new_slots(s)
    cs = s["angles"][slot.clamp(max=s["angles"].shape[0] - 1)]
    k, v, q = _turn(s["Kn"].float(), cs, c), s["Vn"].float(), _turn(s["Q"].float(), cs, c)
    if c["fp8"]:
        k, v = k / s["k_scale"][:, None], v / s["v_scale"][:, None]
        k, v = k.clamp(-448, 448), v.clamp(-448, 448)
    b, t = there.nonzero(as_tuple=True)
    at = slot[b, t]
    page, row = s["block_table"].long()[b, at // c["page"]], at % c["page"]
    _bits(s["K"])[page, row] = _bits(k[b, t].to(s["K"].dtype))
    _bits(s["V"])[page, row] = _bits(v[b, t].to(s["V"].dtype))
    s["Qr"][b, t] = q[b, t].bfloat16()
    return [s["K"], s["V"], s["Qr"]]


def _evict(s):
    c = s["case"]
    B, Hkv, W = s["weights"].shape
    keep = c["sink"] + c["recent"] + c["heavy"]
    if own:
        import paper_2605_11744_b200 as sa
        idx, n, shift, w = sa.kv_evict(s["weights"], s["K"], s["V"], s["block_table"], s["kv_len"], s["dst_table"], sink=c["sink"],
                                       recent=c["recent"], heavy=c["heavy"])
        return [idx, n, shift, w, s["K"], s["V"]]
    n = s["kv_len"].long()[:, None]
    j = torch.arange(W, device="cuda")
    must = (j < c["sink"]) | ((j >= n - c["recent"]) & (j < n))
    worth = s["weights"].masked_fill(must[:, None], math.inf).masked_fill((j >= n)[:, None], -math.inf)
    best = worth.sort(dim=-1, descending=True, stable=True)[1][..., :keep]
    best = torch.where(best < n[..., None], best, W).sort(-1)[0]                      # ascending, what is not there last
    if best.shape[-1] < keep:
        best = torch.cat([best, best.new_full((B, Hkv, keep - best.shape[-1]), W)], -1)
    there = best < W
    b, h, r = there.nonzero(as_tuple=True)
    src = best[b, h, r]
    page, to = s["block_table"].long()[b, src // c["page"]], s["dst_table"].long()[b, r // c["page"]]
    K, V = _bits(s["K"]), _bits(s["V"])
    K[to, r % c["page"], h] = K[page, src % c["page"], h]
    V[to, r % c["page"], h] = V[page, src % c["page"], h]
    w = torch.zeros_like(s["weights"])
    w[b, h, r] = s["weights"][b, h, src]
    count = n[:, 0].clamp(max=keep)
    return [torch.where(there, best, -1).int(), count.int(), (n[:, 0] - count).int(), w, s["K"], s["V"]]


def _rope(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        return sa.rope_rotate(s["X"], s["table"], positions=s["positions"], layout=c["pairs"], inverse=c["inverse"])
    return _turn(s["X"].float(), s["table"][s["positions"].long()], c, c["inverse"]).bfloat16()


# ---- the work no implementation can do without ------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "rope":
        rows = c["B"] * c["L"]
        return {"bytes": rows * (2 * 2 * c["H"] * c["d"] + 4) + 4 * c["rot"] * min(rows, c["L"] + 1000), "flops": 3 * rows * c["H"] * c["rot"]}
    n, new = _lengths(c)
    B, Hkv, d, e = c["B"], c["Hkv"], c["d"], 1 if c["fp8"] else 2
    pages = sum(-(-x // c["page"]) for x in n)
    if c["op"] == "append":
        rows = sum(new)
        return {"bytes": rows * d * (4 * c["Hq"] + 2 * Hkv * (2 + e)) + 4 * c["rot"] * min(rows, max(n)) + 4 * min(pages, rows) + 4 * B,
                "flops": 3 * rows * (c["Hq"] + Hkv) * c["rot"]}
    if c["op"] == "evict":
        kept = [min(x, c["sink"] + c["recent"] + c["heavy"]) for x in n]
        budget = c["sink"] + c["recent"] + c["heavy"]
        W = max(-(-x // c["page"]) for x in n) * c["page"]
        return {"bytes": Hkv * (4 * sum(n) + 4 * B * budget + 4 * B * W + sum(kept) * 4 * d * e) + 4 * pages, "flops": Hkv * sum(n)}
    group = c["Hq"] // Hkv
    rows = keys = pairs = 0
    for x, m in zip(n, new):
        rows += m
        for past in _classes(c):
            low = [0 if past else max(0, p // c["S"] * c["S"] - c["T"]) for p in range(x - m, x)]
            keys += x - min(low)
            pairs += group * sum(p + 1 - lo for p, lo in zip(range(x - m, x), low))
    return {"bytes": 2 * keys * d * e + rows * c["Hq"] * (4 * d + 4) + 4 * pages + 4 * B + (8 * Hkv * sum(n) if c["weights"] else 0),
            "flops": 4 * pairs * d}


# ---- the definitions in 64 bits, one sequence at a time -------------------------------------------------------------------

def _spin(x, table, at, c, inverse):
    """Rows x [L, H, d] turned as complex numbers by the table's rows `at`."""
    r = c["rot"]
    z = torch.view_as_complex(table[at].double().contiguous())[:, None]
    z = z.conj() if inverse else z
    y = x.double().clone()
    if c["pairs"] == "half":
        y[..., :r] = torch.view_as_real(torch.complex(y[..., :r // 2], y[..., r // 2:r]) * z).movedim(-1, -2).flatten(-2)
    else:
        y[..., :r] = torch.view_as_real(torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * z).flatten(-2)
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return torch.stack([_spin(s["X"][b], s["table"], s["positions"][b].long(), c, c["inverse"]) for b in range(c["B"])])
    n, new = _lengths(c)
    page = c["page"]
    if c["op"] == "evict":
        # whole numbers are compared with the plain form's; the moved rows and weights follow from the choice, made here in numpy
        K, V, w = s["K"].double(), s["V"].double(), torch.zeros_like(s["weights"], dtype=torch.float64)
        for b in range(c["B"]):
            for h in range(c["Hkv"]):
                have = s["weights"][b, h, :n[b]].double().cpu().numpy()
                mid = np.arange(min(c["sink"], n[b]), max(min(c["sink"], n[b]), n[b] - c["recent"]))
                mid = mid[np.lexsort((mid, -have[mid]))][:c["heavy"]]
                stay = set(range(min(c["sink"], n[b]))) | set(range(max(0, n[b] - c["recent"]), n[b])) | set(mid.tolist())
                src = torch.tensor(sorted(stay), device="cuda")
                spare = torch.tensor(sorted(set(range(n[b])) - stay), dtype=torch.long, device="cuda")
                if len(src) < min(n[b], c["sink"] + c["recent"] + c["heavy"]):   # sink and recent overlap: the budget goes to the best left
                    more = spare[torch.argsort(-s["weights"][b, h, spare], stable=True)]
                    src = torch.cat([src, more[:min(n[b], c["sink"] + c["recent"] + c["heavy"]) - len(src)]]).sort()[0]
                r = torch.arange(len(src), device="cuda")
                a, z = s["block_table"][b, src // page].long(), s["dst_table"][b, r // page].long()
                K[z, r % page, h], V[z, r % page, h] = K[a, src % page, h], V[a, src % page, h]
                w[b, h, :len(src)] = s["weights"][b, h, src].double()
        return [None, None, None, w, K, V]
    if c["op"] == "append":
        Q = s["Qr"].double()
        K, V = s["K"].double(), s["V"].double()
        for b in range(c["B"]):
            at = torch.arange(n[b] - new[b], n[b], device="cuda")
            Q[b, :new[b]] = _spin(s["Q"][b, :new[b]], s["angles"], at, c, False)
            k, v = _spin(s["Kn"][b, :new[b]], s["angles"], at, c, False), s["Vn"][b, :new[b]].double()
            if c["fp8"]:
                k = (k / s["k_scale"].double()[:, None]).clamp(-448, 448)
                v = (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
            K[s["block_table"][b, at // page].long(), at % page] = k
            V[s["block_table"][b, at // page].long(), at % page] = v
        return [K, V, Q]
    G, d = c["Hq"] // c["Hkv"], c["d"]
    O, lse = s["O"].double(), s["LSE"].double()
    w = s["weights_out"].double() if c["weights"] else None
    for b in range(c["B"]):
        at = torch.arange(n[b], device="cuda")
        pick = s["block_table"][b, at // page].long(), at % page
        K, V = (x.view(torch.uint8)[pick].view(x.dtype).double() for x in (s["K"], s["V"]))
        if c["fp8"]:
            K, V = K * s["k_scale"].double()[:, None], V * s["v_scale"].double()[:, None]
        if c["weights"]:
            w[b, :, :n[b]] = s["weights"][b, :, :n[b]].double()
        for t in range(new[b]):
            p = n[b] - new[b] + t
            for h, past in enumerate(_classes(c)):
                low = 0 if past else max(0, p // c["S"] * c["S"] - c["T"])
                x = s["Q"][b, t, h * G:(h + 1) * G].double() @ K[low:p + 1, h].T / math.sqrt(d)
                lse[b, h * G:(h + 1) * G, t] = torch.logsumexp(x, -1)
                prob = torch.softmax(x, -1)
                O[b, t, h * G:(h + 1) * G] = prob @ V[low:p + 1, h]
                if c["weights"]:
                    w[b, h, low:p + 1] += prob.sum(0)
    return [O, lse] + ([w] if c["weights"] else [])
