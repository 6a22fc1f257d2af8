"""Operators that let a decoding loop run on the GPU by itself and read less of a long cache: what is measured, and their plain
forms.  The cache is that of perf/operators.py: K and V pages [n_pages, page_size, Hkv, d], a block table [B, max_pages], lengths.

  pages      block tables, lengths, slot maps and positions from the lengths that requests ask for, pages from a free list
  append     new rows, keys rotated, into a cache in 8 bits with a scale for each block of rows and head
  decode     attention of each sequence's newest tokens over such a cache, under the segment mask of the head's class
  summarise  the mean key of every block that new rows have filled, in 8 bits with a scale
  select     the blocks of a row's far past that those means score highest, for the heads that read their past
  attend     attention over the chosen blocks and the row's own segment and tail
"""
import math
import random

import torch

own = False   # false: the plain forms below; true: the calls a user makes of the framework


def listed():
    return [
        # a serving batch's decoding step: most sequences grow by a token, some are finished, one is new
        dict(name="pages_step", op="pages", B=64, lo=1, hi=8000, Lq=1, grow=0.9, page=16),
        # prompts of up to 8192 tokens are admitted while others finish
        dict(name="pages_prompts", op="pages", B=48, lo=1, hi=20000, Lq=8192, grow=0.7, page=64),
        # one new token for each sequence of a serving batch; a scale now and then has to be raised
        dict(name="append_tokens_scaled", op="append", B=64, lo=100, hi=8000, Lq=1, Hq=32, Hkv=8, d=128, rot=128, pairs="half", page=64, rows=64),
        # a prompt chunk for three sequences
        dict(name="append_chunk_scaled", op="append", B=3, lo=4500, hi=9001, Lq=4096, Hq=32, Hkv=8, d=128, rot=128, pairs="half", page=64, rows=64),
        # one user's short chat turn
        dict(name="decode_short_scaled", op="decode", B=1, lo=517, hi=517, Lq=1, Hq=32, Hkv=8, d=128, S=2048, T=512, past=2, page=16, rows=16),
        # the 128K configuration, every second head with its whole past
        dict(name="decode_128k_scaled", op="decode", B=8, lo=100000, hi=131072, Lq=1, Hq=32, Hkv=8, d=128, S=8192, T=2048, past=4, page=128,
             rows=64),
        # a decoding step in which a few sequences fill a block
        dict(name="summarise_step", op="summarise", B=64, lo=100, hi=30000, Lq=1, Hkv=8, d=128, page=64, block=64, scaled=False),
        # the prompts of a batch, once their rows are in an 8-bit cache
        dict(name="summarise_prompts", op="summarise", B=8, lo=16000, hi=65536, Lq=65536, Hkv=8, d=128, page=128, block=64, scaled=True),
        # one sequence of 16K
        dict(name="select_one", op="select", B=1, lo=16100, hi=16100, Lq=1, Hq=32, Hkv=8, d=128, S=2048, T=512, past=2, page=64, block=64, n=16,
             sink=1),
        # a batch of 128K sequences, every second head
        dict(name="select_128k", op="select", B=16, lo=90000, hi=131072, Lq=1, Hq=32, Hkv=8, d=128, S=4096, T=1024, past=4, page=64, block=32, n=64,
             sink=1),
        # one sequence of 16K, the same blocks
        dict(name="attend_one", op="attend", B=1, lo=16100, hi=16100, Lq=1, Hq=32, Hkv=8, d=128, S=2048, T=512, past=2, page=64, block=64, n=16,
             rows=0),
        # a batch of 128K sequences in 8 bits, four tokens at a time (a draft to be checked)
        dict(name="attend_128k_scaled", op="attend", B=16, lo=90000, hi=131072, Lq=4, Hq=32, Hkv=8, d=128, S=2048, T=512, past=8, page=64, block=64, n=64,
             rows=64),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["pages", "append", "append", "decode", "decode", "summarise", "select", "attend", "attend"])
    d, Hkv, B = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), _log(rng, 1, 48)
    rows = rng.choice([16, 32, 64, 128])
    page = rows * rng.choice([1, 2, 3, 4])
    if op == "pages":
        return dict(op=op, B=_log(rng, 5, 300), lo=1, hi=_log(rng, 100, 30000), Lq=_log(rng, 1, 6000), grow=rng.uniform(0.5, 1),
                    page=rng.choice([1, 8, 16, 100, 128]))
    if op == "append":
        Lq = _log(rng, 1, 12000 // B)
        return dict(op=op, B=B, lo=Lq, hi=Lq + _log(rng, 1, 4000), Lq=Lq, Hq=Hkv * rng.choice([1, 2, 4]), Hkv=Hkv, d=d, rot=rng.choice([16, 32, 48, 64, d]),
                    pairs=rng.choice(["half", "interleaved"]), page=page, rows=rows)
    hi = _log(rng, 1, min(131072, 300000 // B))
    lo = max(1, int(hi * rng.random()))
    S = _log(rng, 64, 8192)
    if op == "decode":
        return dict(op=op, B=B, lo=lo, hi=hi, Lq=rng.choice([1, 1, 1, 2, 5]), Hq=Hkv * rng.choice([1, 2, 3, 4, 8]), Hkv=Hkv, d=d, S=S, T=rng.randint(0, S),
                    past=rng.randint(0, Hkv), page=page, rows=rows)
    if op == "summarise":
        return dict(op=op, B=B, lo=lo, hi=hi, Lq=_log(rng, 1, hi), Hkv=Hkv, d=d, page=page, block=rows, scaled=rng.random() < 0.5)
    # long enough that the longest sequence has more blocks behind its segment and tail than are chosen
    hi = _log(rng, 1000, max(1000, min(131072, 300000 // B)))
    S = _log(rng, 64, hi // 8)
    n = _log(rng, 1, max(1, min(100, 4096 // rows, hi // (2 * rows))))
    c = dict(op=op, B=B, lo=max(1, int(hi * rng.random())), hi=hi, Lq=rng.choice([1, 1, 1, 2, 4]), Hq=Hkv * rng.choice([1, 2, 4, 8]), Hkv=Hkv, d=d,
             S=S, T=rng.randint(0, S), past=rng.randint(1, Hkv), page=page, block=rows, n=n)
    return dict(c, sink=rng.randint(0, min(2, n))) if op == "select" else dict(c, rows=rng.choice([0, 16, rows]))


def _lengths(c):
    """The sequences' lengths, and how many tokens of each are new (a case's own, whatever the seed)."""
    r = random.Random("%d %d %d" % (c["B"], c["lo"], c["hi"]))
    n = [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])]
    n[-1] = c["hi"]
    return n, [min(x, c["Lq"]) for x in n]


def _wanted(c):
    """The lengths that requests ask for: most grow by up to Lq, some end or give rows back."""
    r = random.Random("%d %d %d %d" % (c["B"], c["lo"], c["hi"], c["Lq"]))
    n = [r.randint(c["lo"], c["hi"]) if r.random() > 0.1 else 0 for _ in range(c["B"])]
    want = [x + (c["Lq"] if c["Lq"] < 8 else r.randint(1, c["Lq"])) if r.random() < c["grow"] else r.choice([0, x, max(0, x - r.randint(1, 8))]) for x in n]
    return n, want


def _classes(c):
    # `past` of the KV heads read their past, spread over the heads; the others their segment and its carried tail
    return [int((h * c["past"]) // c["Hkv"] != ((h + 1) * c["past"]) // c["Hkv"]) for h in range(c["Hkv"])]


def _angles(n_pos, rot):
    w = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * w
    return torch.stack([a.cos(), a.sin()], -1).float()


def prepare(case, seed):
    c, s = case, dict(case=case)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    B, page = c["B"], c["page"]
    n, ask = _wanted(c) if c["op"] == "pages" else (_lengths(c)[0],) * 2
    need = [-(-x // page) for x in n]
    per = max(-(-max(x, y) // page) for x, y in zip(n, ask))
    spare = sum(max(0, -(-y // page) - x) for x, y in zip(need, ask))
    spare -= spare // 8 if c["op"] == "pages" else 0      # the last of the queue may have to wait
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").int()      # pages are handed out in no order
    table = torch.full((B, per), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    s["block_table"], s["kv_len"] = table, ints(n)
    if c["op"] == "pages":
        s["want"], s["shift"] = ints(ask), torch.randint(0, 50, (B,), generator=g, device="cuda").int()
        s["free"], s["count"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda"), ints([spare])
        s["free"][:spare] = order[at:]
        return s
    new = [min(x, c["Lq"]) for x in n]
    s["q_len"] = ints(new) if min(new) < c["Lq"] else None
    Hkv, d = c["Hkv"], c["d"]
    if c["op"] == "select":
        s["Q"], s["mask"] = normal(B, c["Lq"], c["Hq"], d), _classes(c)
        s["sums"] = torch.randint(-127, 128, (pages, page // c["block"], Hkv, d), generator=g, device="cuda").to(torch.int8)
        s["sum_scale"] = (0.5 + torch.rand((pages, page // c["block"], Hkv), generator=g, device="cuda")) / 300
        s["idx"] = torch.full((B, c["Lq"], Hkv, c["n"]), -1, dtype=torch.int32, device="cuda")
        return s
    s["K"] = normal(pages, page, Hkv, d)
    s["V"] = normal(pages, page, Hkv, d) if c["op"] != "summarise" else s["K"]
    rows = c.get("rows", c.get("block") if c.get("scaled") else 0)
    s["k_scale"] = s["v_scale"] = None
    if rows:
        # each block's largest value is near 448 times its scale, as an append leaves it; scales differ by a few powers of two
        s["K"], s["V"] = ((80 * s[x]).clamp(-448, 448).to(torch.float8_e4m3fn) for x in "KV")
        s["k_scale"], s["v_scale"] = (torch.exp2(torch.randint(-8, -5, (pages, page // rows, Hkv), generator=g, device="cuda").float()) for _ in range(2))
    if c["op"] == "summarise":
        s["sums"] = torch.zeros((pages, page // c["block"], Hkv, d), dtype=torch.int8, device="cuda")
        s["sum_scale"] = torch.zeros((pages, page // c["block"], Hkv), device="cuda")
        return s
    s["Q"] = normal(B, c["Lq"], c["Hq"], d)
    if c["op"] == "append":
        # rows of keys differ in size, so that a block's scale is at times raised
        size = torch.exp2(torch.randint(-2, 1, (B, c["Lq"], 1, 1), generator=g, device="cuda").float()).bfloat16()
        s["Kn"], s["Vn"] = normal(B, c["Lq"], Hkv, d) * size, normal(B, c["Lq"], Hkv, d) * size
        s["Qr"], s["angles"] = torch.zeros_like(s["Q"]), _angles(max(n), c["rot"])
        return s
    s["mask"], s["O"], s["LSE"] = _classes(c), torch.zeros_like(s["Q"]), torch.zeros((B, c["Hq"], c["Lq"]), device="cuda")
    if c["op"] == "attend":
        # as a selection leaves them: ascending, then -1
        room = _window(s)[0][..., None, None] // c["block"]      # [B, Lq, 1, 1]
        score = torch.rand((B, c["Lq"], Hkv, max(1, c["hi"] // c["block"])), generator=g, device="cuda")
        score = score.masked_fill(torch.arange(score.shape[-1], device="cuda") >= room, -1.0)
        top, idx = score.topk(min(c["n"], score.shape[-1]))
        idx = torch.where(top >= 0, idx, 1 << 30).sort(-1)[0]
        idx = torch.where(idx < 1 << 30, idx, -1)
        s["idx"] = torch.nn.functional.pad(idx, (0, c["n"] - idx.shape[-1]), value=-1).int()
        past = torch.tensor(s["mask"], device="cuda").bool()
        s["idx"] = torch.where(past[:, None], s["idx"], torch.full_like(s["idx"], -1)).contiguous()
    return s


def run(s):
    return {"pages": _pages, "append": _append, "decode": _decode, "summarise": _summarise, "select": _select, "attend": _attend}[s["case"]["op"]](s)


# ---- plain forms, in 32 bits ----------------------------------------------------------------------------------------

def _pages(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        n, count, q, slots, pos = sa.pages_resize(s["want"], s["block_table"], s["kv_len"], s["free"], s["count"], c["page"], c["Lq"], pos_shift=s["shift"])
        return [n, count, q, slots, pos, s["block_table"], s["free"]]
    page, table = c["page"], s["block_table"]
    n, want = s["kv_len"].long(), s["want"].long()
    have, need = (n + page - 1) // page, (want + page - 1) // page
    back, take = (have - need).clamp(min=0), (need - have).clamp(min=0)
    sure = s["count"].long() + back.sum()                          # pages there are, those given back among them, on top
    served = (take == 0) | (take.cumsum(0) <= sure)                # first come, first served
    take = torch.where(served, take, 0)
    n_out = torch.where(served, want, n)
    k = torch.arange(table.shape[1], device="cuda")
    gives = (k >= need[:, None]) & (k < have[:, None])
    stack = torch.cat([s["free"][:s["count"].long().sum()].long(), table[gives].long()])
    b, i = ((k >= have[:, None]) & (k < (have + take)[:, None])).nonzero(as_tuple=True)
    table[b, i] = stack.flip(0)[:len(b)].int()
    left = stack[:len(stack) - len(b)]
    s["free"][:len(left)] = left.int()
    grown = (n_out - n).clamp(min=0)
    t = torch.arange(c["Lq"], device="cuda")
    there = t < grown[:, None]
    slot = torch.where(there, n[:, None] + t, 0)
    where = table.long().gather(1, slot // page) * page + slot % page
    return [n_out.int(), torch.tensor([1], device="cuda").int() * len(left), grown.int(), torch.where(there, where, -1),
            torch.where(there, slot + s["shift"].long()[:, None], 0).int(), table, s["free"]]


def _new_slots(s):
    """Slot of every new row [B, Lq] and whether the row is there at all."""
    c, n = s["case"], s["kv_len"].long()
    t = torch.arange(c["Lq"], device="cuda")
    new = n.clamp(max=c["Lq"]) if s["q_len"] is None else s["q_len"].long()
    return (n - new)[:, None] + t, t < new[:, None]


def _bits(x):
    # 8-bit values are moved as bytes
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _at(s, slot):
    """Page and row of slots [B, ...]."""
    page = s["case"]["page"]
    flat = (slot // page).clamp(0, s["block_table"].shape[1] - 1).flatten(1)
    return s["block_table"].long().clamp(min=0).gather(1, flat).view(slot.shape), slot % page


def _rows(s, name, scale, slot):
    """The cache's rows at slots [B, X] as 32-bit values [B, X, Hkv, d]."""
    page, row = _at(s, slot)
    x = _bits(s[name])[page, row].view(s[name].dtype).float()
    return x if s[scale] is None else x * s[scale][page, row // s["case"]["rows"]][..., None]


def _turn(x, cs, c):
    """x [B, L, H, d] in 32 bits rotated by cs [B, L, rot/2, 2]."""
    r = c["rot"]
    cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["pairs"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([y, z], -1) if c["pairs"] == "half" else torch.stack([y, z], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _store(s, name, scale, x):
    """New rows x [B, Lq, Hkv, d] in 8 bits, with the scales of the blocks they fall into."""
    c, rows = s["case"], s["case"]["rows"]
    pages, scales = s[name], s[scale]
    slot, there = _new_slots(s)
    first = slot[:, :1]
    block = torch.where(there, slot // rows - first // rows, 0)                                  # of those touched
    some = (c["Lq"] + rows - 2) // rows + 1
    top = x.abs().amax(-1).masked_fill(~there[..., None], 0.0)
    most = torch.zeros((c["B"], some, c["Hkv"]), device="cuda").scatter_reduce(1, block[..., None].expand_as(top), top, "amax")
    m, e = torch.frexp(most)                                                                     # m 2^e, 0.5 <= m < 1
    e = torch.where(most > 0, e.long() - 9 + (m > 0.875), -40).clamp(-40, 119)
    need = torch.ldexp(torch.ones_like(most), e)
    start = (first // rows + torch.arange(some, device="cuda")) * rows                           # [B, some]
    b, k = ((start < s["kv_len"].long()[:, None]) & there[:, :1]).nonzero(as_tuple=True)
    page, row = _at(s, start)
    old = torch.where((start < first)[..., None], scales[page, row // rows], 0.0)
    got = torch.maximum(old, need)
    # rows that were there already, of the first block, where its scale has grown
    j = start[:, :1] + torch.arange(rows, device="cuda")
    b0, j0, h0 = ((j < first)[..., None] & (got > old)[:, :1] & there[:, :1, None]).nonzero(as_tuple=True)
    pj, rj = _at(s, j)
    pj, rj = pj[b0, j0], rj[b0, j0]
    was = _bits(pages)[pj, rj, h0].view(pages.dtype).float() * (old[b0, 0, h0] / got[b0, 0, h0])[:, None]
    _bits(pages)[pj, rj, h0] = _bits(was.to(pages.dtype))
    scales[page[b, k], row[b, k] // rows] = got[b, k]
    b, t = there.nonzero(as_tuple=True)
    y = (x[b, t] / got[b, block[b, t]][..., None]).clamp(-448, 448)
    page, row = _at(s, slot.clamp(min=0))
    _bits(pages)[page[b, t], row[b, t]] = _bits(y.to(pages.dtype))


def _append(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        sa.kv_append(s["Kn"], s["Vn"], s["K"], s["V"], s["block_table"], s["kv_len"], table=s["angles"], layout=c["pairs"], Q=s["Q"],
                     q_out=s["Qr"], q_len=s["q_len"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return [s["K"], s["V"], s["k_scale"], s["v_scale"], s["Qr"]]
    slot, there = _new_slots(s)
    cs = s["angles"][slot.clamp(0, s["angles"].shape[0] - 1)]
    _store(s, "K", "k_scale", _turn(s["Kn"].float(), cs, c))
    _store(s, "V", "v_scale", s["Vn"].float())
    q = _turn(s["Q"].float(), cs, c).bfloat16()
    s["Qr"].copy_(torch.where(there[..., None, None], q, s["Qr"]))
    return [s["K"], s["V"], s["k_scale"], s["v_scale"], s["Qr"]]


def _softmax_over(s, x, V, pattern, there):
    """O and LSE from scores x [B, Hkv, g, Lq, X] (-inf: not visible), rows that are not there as they were."""
    c = s["case"]
    m = x.amax(-1, keepdim=True)
    e = (x - m.masked_fill(m == -math.inf, 0.0)).exp()
    z = e.sum(-1, keepdim=True)
    lse = (m + z.log()).squeeze(-1).reshape(c["B"], c["Hq"], c["Lq"])
    P = e / z.masked_fill(z == 0, 1.0)
    O = torch.einsum(pattern, P, V).reshape(s["Q"].shape).bfloat16()
    return [torch.where(there[:, :, None, None], O, s["O"]), torch.where(there[:, None], lse, s["LSE"])]


def _decode(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        return list(sa.seg_attn_decode(s["Q"], s["K"], s["V"], s["block_table"], s["kv_len"], c["S"], c["T"], s["mask"], q_len=s["q_len"],
                                       k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["O"], lse=s["LSE"]))
    p, there = _new_slots(s)
    j = torch.arange(s["block_table"].shape[1] * c["page"], device="cuda")
    low = (p // c["S"] * c["S"] - c["T"]).clamp(min=0)[:, None] * (1 - torch.tensor(s["mask"], device="cuda"))[None, :, None]
    sees = (j >= low[..., None]) & (j <= p[:, None, :, None]) & there[:, None, :, None]                     # [B, Hkv, Lq, slots]
    at = j.expand(c["B"], -1)
    q = s["Q"].float().reshape(c["B"], c["Lq"], c["Hkv"], -1, c["d"])
    x = torch.einsum("btcgd,bjcd->bcgtj", q, _rows(s, "K", "k_scale", at)) * c["d"] ** -0.5
    x = x.masked_fill(~sees[:, :, None], -math.inf)
    return _softmax_over(s, x, _rows(s, "V", "v_scale", at), "bcgtj,bjcd->btcgd", there)


def _summarise(s):
    c, block = s["case"], s["case"]["block"]
    if own:
        import paper_2605_11744_b200 as sa
        sa.blocks_summarise(s["K"], s["block_table"], s["kv_len"], c["Lq"], s["sums"], s["sum_scale"], q_len=s["q_len"], k_scale=s["k_scale"])
        return [s["sums"], s["sum_scale"]]
    slot, there = _new_slots(s)
    some = (c["Lq"] + block - 2) // block + 1
    k = slot[:, :1] // block + torch.arange(some, device="cuda")
    b, i = (((k + 1) * block <= s["kv_len"].long()[:, None]) & there[:, :1]).nonzero(as_tuple=True)         # blocks that are full
    page, row = _at(s, k * block)
    page, row = page[b, i], row[b, i]
    at = page[:, None], row[:, None] + torch.arange(block, device="cuda")
    x = _bits(s["K"])[at].view(s["K"].dtype).double()                                                      # [blocks, rows, Hkv, d]
    if s["k_scale"] is not None:
        x = x * s["k_scale"][page, row // block].double()[:, None, :, None]
    mean = (x.sum(1) / block).float()
    scale = mean.abs().amax(-1) / 127.0
    q = (mean / scale[..., None]).round().nan_to_num(0.0)
    s["sums"][page, row // block] = q.to(torch.int8)
    s["sum_scale"][page, row // block] = scale
    return [s["sums"], s["sum_scale"]]


def _window(s):
    """For each new row [B, Lq]: where the part that it sees in whole begins for heads with a past and for the others."""
    c = s["case"]
    low = (_new_slots(s)[0] // c["S"] * c["S"] - c["T"]).clamp(min=0)
    return low // c["block"] * c["block"], low


def _select(s):
    c = s["case"]
    if own:
        import paper_2605_11744_b200 as sa
        return sa.blocks_select(s["Q"], s["sums"], s["sum_scale"], s["block_table"], s["kv_len"], c["page"], c["S"], c["T"], c["n"], sink=c["sink"],
                                head_past_mask=s["mask"], q_len=s["q_len"], out=s["idx"])
    B, Lq, Hkv = c["B"], c["Lq"], c["Hkv"]
    q = s["Q"].double().reshape(B, Lq, Hkv, -1, c["d"]).sum(3).float()
    size = q.abs().amax(-1, keepdim=True) / 127.0
    q = (q / size).round().nan_to_num(0.0)
    k = torch.arange(s["block_table"].shape[1] * (c["page"] // c["block"]), device="cuda")
    page, row = _at(s, (k * c["block"]).expand(B, -1))
    at = page, row // c["block"]
    # whole numbers below 2^24: the sums are exact
    score = torch.einsum("btcd,bjcd->btcj", q, s["sums"][at].float()) * s["sum_scale"][at].transpose(1, 2)[:, None]
    room = _window(s)[0] // c["block"]
    score = score.masked_fill(k < c["sink"], math.inf).masked_fill((k >= room[..., None])[:, :, None], -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True)[1][..., :c["n"]]
    best = torch.where(best < room[..., None, None], best, len(k)).sort(-1)[0]
    best = torch.nn.functional.pad(best, (0, max(0, c["n"] - best.shape[-1])), value=len(k))
    past = torch.tensor(s["mask"], device="cuda").bool()[:, None]
    best = torch.where((best < len(k)) & past, best, -1).int()
    return torch.where(_new_slots(s)[1][..., None, None], best, s["idx"])


def _attend(s):
    c, block = s["case"], s["case"]["block"]
    if own:
        import paper_2605_11744_b200 as sa
        return list(sa.seg_attn_decode(s["Q"], s["K"], s["V"], s["block_table"], s["kv_len"], c["S"], c["T"], s["mask"], q_len=s["q_len"],
                                       k_scale=s["k_scale"], v_scale=s["v_scale"], blocks=s["idx"], block=block, out=s["O"], lse=s["LSE"]))
    B, Lq, Hkv, d = c["B"], c["Lq"], c["Hkv"], c["d"]
    p, there = _new_slots(s)
    past = torch.tensor(s["mask"], device="cuda").bool()
    whole, low = _window(s)
    low = torch.where(past, whole[..., None], low[..., None])                                               # [B, Lq, Hkv]
    far = (s["idx"].long()[..., None] * block + torch.arange(block, device="cuda")).flatten(-2)
    near = low[..., None] + torch.arange(min(c["hi"], c["S"] + c["T"] + block), device="cuda")
    at = torch.cat([far, near], -1)                                                                         # [B, Lq, Hkv, X]
    sees = torch.cat([far >= 0, near <= p[..., None, None]], -1) & there[..., None, None]
    at = at.clamp(0, s["block_table"].shape[1] * c["page"] - 1)
    page, row = _at(s, at)
    h = torch.arange(Hkv, device="cuda")[:, None]

    def rows(name, scale):
        x = _bits(s[name])[page, row, h].view(s[name].dtype).float()
        return x if s[scale] is None else x * s[scale][page, row // c["rows"], h][..., None]

    q = s["Q"].float().reshape(B, Lq, Hkv, -1, d)
    x = torch.einsum("btcgd,btcjd->bcgtj", q, rows("K", "k_scale")) * d ** -0.5
    x = x.masked_fill(~sees.permute(0, 2, 1, 3)[:, :, None], -math.inf)
    return _softmax_over(s, x, rows("V", "v_scale"), "bcgtj,btcjd->btcgd", there)


# ---- the work no implementation can do without ------------------------------------------------------------------------

def work(case):
    c, page = case, case["page"]
    B = c["B"]
    if c["op"] == "pages":
        n, want = _wanted(c)
        moved = sum(abs(-(-x // page) + (-y // page)) for x, y in zip(n, want))
        return {"bytes": 8 * moved + 12 * B * c["Lq"] + 20 * B + 8, "flops": 4 * B}
    n, new = _lengths(c)
    Hkv, d = c["Hkv"], c["d"]
    rows, pages = sum(new), sum(-(-x // page) for x in n)
    if c["op"] == "append":
        blocks = sum((x - 1) // c["rows"] - (x - m) // c["rows"] + 1 for x, m in zip(n, new))
        return {"bytes": rows * d * (4 * c["Hq"] + 2 * Hkv * 3) + 4 * c["rot"] * min(rows, max(n)) + blocks * (8 * Hkv + 4) + 4 * B,
                "flops": rows * d * (3 * (c["Hq"] + Hkv) + 4 * Hkv)}
    if c["op"] == "summarise":
        full = sum(x // c["block"] - (x - m) // c["block"] for x, m in zip(n, new))
        e = 1 if c["scaled"] else 2
        return {"bytes": full * (Hkv * (c["block"] * d * e + d + 4 + 4 * (2 - e)) + 4) + 4 * B, "flops": full * Hkv * d * (c["block"] + 3)}
    past = sum(_classes(c))
    if c["op"] == "decode":
        keys = blocks = pairs = 0
        for x, m in zip(n, new):
            for kind in _classes(c):
                low = [0 if kind else max(0, p // c["S"] * c["S"] - c["T"]) for p in range(x - m, x)]
                keys += x - min(low)
                blocks += (x - 1) // c["rows"] - min(low) // c["rows"] + 1
                pairs += c["Hq"] // Hkv * sum(p + 1 - lo for p, lo in zip(range(x - m, x), low))
        return {"bytes": 2 * keys * d + 8 * blocks + rows * c["Hq"] * (4 * d + 4) + 4 * pages + 4 * B, "flops": 4 * pairs * d}
    window = [[max(0, p // c["S"] * c["S"] - c["T"]) for p in range(x - m, x)] for x, m in zip(n, new)]
    if c["op"] == "select":
        most = sum(max(low) // c["block"] for low in window)
        each = sum(lo // c["block"] for low in window for lo in low)
        return {"bytes": most * (past * (d + 4) + 4) + rows * (2 * c["Hq"] * d + 4 * Hkv * c["n"]) + 4 * B, "flops": 2 * each * past * d}
    e = 1 if c["rows"] else 2
    keys = pairs = 0      # a window shared by a sequence's new rows is read once; the blocks that they choose are hardly ever the same
    for x, low in zip(n, window):
        for kind in _classes(c):
            first = min(low) // c["block"] * c["block"] if kind else min(low)
            most = max(low) // c["block"]
            keys += x - first + (min(sum(min(c["n"], lo // c["block"]) for lo in low), most) * c["block"] if kind else 0)
            for p, lo in zip(range(x - len(low), x), low):
                start = lo // c["block"] * c["block"] if kind else lo
                pairs += c["Hq"] // Hkv * (p + 1 - start + (min(c["n"], start // c["block"]) * c["block"] if kind else 0))
    return {"bytes": 2 * keys * d * e + (8 * keys // c["rows"] if c["rows"] else 0) + rows * (c["Hq"] * (4 * d + 4) + 4 * past * c["n"]) + 4 * B,
            "flops": 4 * pairs * d}


# ---- the definitions in 64 bits, one sequence at a time -------------------------------------------------------------------

def _stored(s, c, name, scale, b, at):
    """Rows of sequence b at slots `at` as [rows, Hkv, d]."""
    page = c["page"]
    pick = s["block_table"][b, at // page].long(), at % page
    x = s[name].view(torch.uint8)[pick].view(s[name].dtype).double() if s[scale] is not None else s[name][pick].double()
    return x if s[scale] is None else x * s[scale][pick[0], pick[1] // c.get("rows", c.get("block"))].double()[..., None]


def _spin(x, table, at, c):
    """Rows x [L, H, d] turned as complex numbers by the table's rows `at`."""
    r = c["rot"]
    z = torch.view_as_complex(table[at].double().contiguous())[:, None]
    y = x.double().clone()
    if c["pairs"] == "half":
        y[..., :r] = torch.view_as_real(torch.complex(y[..., :r // 2], y[..., r // 2:r]) * z).movedim(-1, -2).flatten(-2)
    else:
        y[..., :r] = torch.view_as_real(torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * z).flatten(-2)
    return y


def exact(case, seed):
    c = case
    if c["op"] in ("pages", "select"):
        return None      # whole numbers alone
    s = prepare(case, seed)
    n, new = _lengths(c)
    page, Hkv, d = c["page"], c["Hkv"], c["d"]
    if c["op"] == "summarise":
        scale = s["sum_scale"].double()
        for b in range(c["B"]):
            k = torch.arange((n[b] - new[b]) // c["block"], n[b] // c["block"], device="cuda")
            if len(k):
                at = (k[:, None] * c["block"] + torch.arange(c["block"], device="cuda")).flatten()
                mean = _stored(s, c, "K", "k_scale", b, at).view(len(k), c["block"], Hkv, d).mean(1)
                scale[s["block_table"][b, k * c["block"] // page].long(), k * c["block"] % page // c["block"]] = mean.abs().amax(-1) / 127
        return [None, scale]
    if c["op"] == "append":
        # values as multiples of the scales that the block's rows then have, not rounded
        rows, out = c["rows"], [s["K"].double(), s["V"].double(), s["k_scale"].double(), s["v_scale"].double(), s["Qr"].double()]
        for b in range(c["B"]):
            at = torch.arange(n[b] - new[b], n[b], device="cuda")
            out[4][b, :new[b]] = _spin(s["Q"][b, :new[b]], s["angles"], at, c)
            for x, full, scales in ((_spin(s["Kn"][b, :new[b]], s["angles"], at, c), out[0], out[2]), (s["Vn"][b, :new[b]].double(), out[1], out[3])):
                starts = torch.arange((n[b] - new[b]) // rows * rows, n[b], rows, device="cuda")
                pad = int(at[0] - starts[0])
                top = torch.nn.functional.pad(x.abs().amax(-1), (0, 0, pad, len(starts) * rows - pad - len(at))).view(len(starts), rows, Hkv).amax(1)
                where = s["block_table"][b, starts // page].long(), starts % page // rows
                old = scales[where].clone()
                got = torch.exp2((top / 448).log2().ceil().clamp(-40, 119))
                if pad:
                    got[0] = torch.maximum(got[0], old[0])
                    j = torch.arange(int(starts[0]), int(at[0]), device="cuda")
                    full[s["block_table"][b, j // page].long(), j % page] *= (old[0] / got[0])[:, None]
                scales[where] = got
                full[s["block_table"][b, at // page].long(), at % page] = x / got[(at - starts[0]) // rows][..., None]
        return out
    G = c["Hq"] // Hkv
    O, lse = s["O"].double(), s["LSE"].double()
    for b in range(c["B"]):
        at = torch.arange(n[b], device="cuda")
        K, V = _stored(s, c, "K", "k_scale", b, at), _stored(s, c, "V", "v_scale", b, at)
        for t in range(new[b]):
            p = n[b] - new[b] + t
            low = max(0, p // c["S"] * c["S"] - c["T"])
            for h, past in enumerate(_classes(c)):
                sees = (at <= p) & (at >= (low if c["op"] == "attend" or not past else 0))
                if c["op"] == "attend" and past:
                    sees |= (at <= p) & (at >= low - low % c["block"])
                    for k in s["idx"][b, t, h].tolist():
                        if k >= 0:
                            sees[k * c["block"]:(k + 1) * c["block"]] = True
                x = s["Q"][b, t, h * G:(h + 1) * G].double() @ K[sees, h].T / math.sqrt(d)
                lse[b, h * G:(h + 1) * G, t] = torch.logsumexp(x, -1)
                O[b, t, h * G:(h + 1) * G] = torch.softmax(x, -1) @ V[sees, h]
    return [O, lse]
