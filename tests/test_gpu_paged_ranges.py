"""The paged cache's kernels where a block goes through many tiles of several items: rings of stages that wrap, score buffers in
use again, outputs rescaled from tile to tile, values that are not finite hidden in the middle of a range; eviction with more keys
than a block keeps in shared memory; and a captured eviction compared bit by bit."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu


def shared_pages(B, distinct, cap, Hkv, d, page, fp8, seed, trend=0.0, q0=32.0):
    """Pages of `distinct` sequences of cap slots, read by B sequences in turn.  With a trend, element 0 of the keys adds
    trend * slot / 64 to the scores of queries whose element 0 is q0."""
    g = torch.Generator().manual_seed(seed)
    per = -(-cap // page)
    order = torch.randperm(distinct * per, generator=g).reshape(distinct, per)
    k, v = torch.randn(distinct * per, page, Hkv, d, generator=g), torch.randn(distinct * per, page, Hkv, d, generator=g)
    scale = 1.0
    if fp8:
        k, v, scale = 4 * k, 4 * v, 0.25
    slot = torch.arange(per * page).reshape(per, page)
    for s in range(distinct):
        k[order[s], :, :, 0] = (trend * slot / 64 * d ** 0.5 / q0 / scale)[:, :, None].expand(per, page, Hkv)
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    table = order[torch.arange(B) % distinct].int()
    scales = dict(k_scale=torch.full((Hkv,), scale).cuda(), v_scale=torch.full((Hkv,), scale).cuda()) if fp8 else {}
    return k.to(kind).cuda(), v.to(kind).cuda(), table, scales, scale


def decode64(Q, K, V, table, lens, rows, S, T, mask, page, scale):
    """What ref.decode gives, sequence by sequence in 64 bits on the device: O, LSE, sum of p|v|, largest sum of terms, weights."""
    B, Lq, Hq, d = Q.shape
    Hkv, cap = K.shape[2], table.shape[1] * page
    O, spread = np.full((B, Lq, Hq, d), np.nan), np.zeros((B, Lq, Hq, d))
    lse, terms, w = np.full((B, Hq, Lq), np.nan), np.zeros((B, Hq, Lq)), np.zeros((B, Hkv, cap))
    for b in range(B):
        n, m = lens[b], rows[b]
        if m == 0:
            continue
        k, v = (x[table[b].long().cuda()].reshape(-1, Hkv, d)[:n].double() * scale for x in (K.float(), V.float()))
        q = Q[b, :m].double().cuda().reshape(m, Hkv, Hq // Hkv, d)
        s = torch.einsum("thgd,jhd->thgj", q, k) * d ** -0.5
        pos = torch.arange(n - m, n, device="cuda")
        first = torch.stack([torch.zeros_like(pos) if c == 1 else torch.clamp(pos // S * S - (T if c == 0 else 0), min=0) for c in mask])     # [Hkv, m]
        j = torch.arange(n, device="cuda")
        see = (j[None, None] >= first[:, :, None]) & (j[None, None] <= pos[None, :, None])     # [Hkv, m, n]
        s = torch.where(see.transpose(0, 1)[:, :, None], s, -math.inf)
        p = torch.softmax(s, -1)
        O[b, :m] = torch.einsum("thgj,jhd->thgd", p, v).reshape(m, Hq, d).cpu().numpy()
        spread[b, :m] = torch.einsum("thgj,jhd->thgd", p, v.abs()).reshape(m, Hq, d).cpu().numpy()
        lse[b, :, :m] = torch.logsumexp(s, -1).reshape(m, Hq).T.cpu().numpy()
        t = torch.where(see.transpose(0, 1)[:, :, None], torch.einsum("thgd,jhd->thgj", q.abs(), k.abs()) * d ** -0.5, 0.0)
        terms[b, :, :m] = t.amax(-1).reshape(m, Hq).T.cpu().numpy()
        w[b, :, :n] = p.sum((0, 2)).cpu().numpy()
    return O, lse, spread, terms, w


# new rows, query heads to a KV head (their product: rows of a KV head), head dimension, 8-bit cache
RANGES = [(2, 4, 128, False), (4, 4, 64, False), (8, 4, 64, False), (8, 4, 128, False), (9, 4, 64, False), (16, 4, 64, False), (16, 4, 128, False),
          (32, 4, 64, False), (32, 4, 128, False), (40, 4, 128, False), (2, 4, 64, True), (4, 4, 128, True), (8, 4, 64, True), (8, 4, 128, True),
          (16, 4, 64, True), (16, 4, 128, True), (32, 4, 128, True)]
B, S, T, PAGE, MASK = 192, 1024, 256, 32, [0, 1]


def batch(Lq, g, d, fp8, trend, seed):
    """192 sequences whose new rows lie across the border between the second and the third segment: a local head's first rows see
    768 and on, the last ones 1792 and on, heads with their past everything.  At least 16 tiles to each of 148 x 2 blocks."""
    K, V, table, scales, scale = shared_pages(B, 12, 2048 + 64, 2, d, PAGE, fp8, seed, trend)
    gen = torch.Generator().manual_seed(seed + 1)
    Q = torch.randn(B, Lq, 2 * g, d, generator=gen)
    Q[..., 0] = 32.0
    lens = [2048 + (5 * b) % Lq + (1 if Lq == 1 else 0) for b in range(B)]
    rows = [Lq - (b % 3 if b % 11 == 0 else 0) for b in range(B)]
    rows[7], rows[100] = 0, 1 if Lq > 1 else 0
    return K, V, table, scales, scale, Q.bfloat16(), lens, rows


def run(Q, K, V, table, scales, lens, rows, **kw):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return sa.seg_attn_decode(Q.cuda(), K, V, table.cuda(), i32(lens), S, T, MASK, q_len=i32(rows), **scales, **kw)


def test_the_reference_on_the_device_is_the_reference():
    K, V, table, scales, scale, Q, lens, rows = batch(3, 2, 64, True, 2.0, seed=3)
    some = [0, 1, 7, 11, 22]
    pick = lambda x: [x[b] for b in some]
    a = decode64(Q[some], K, V, table[some], pick(lens), pick(rows), S, T, MASK, PAGE, scale)
    ks = np.full(2, scale)
    z = ref.decode(Q[some].float().double().numpy(), K, V, table[some].numpy(), pick(lens), pick(rows), S, T, MASK, 64 ** -0.5, PAGE, k_scale=ks, v_scale=ks)
    for x, y in zip(a, z):
        assert np.array_equal(np.isnan(x), np.isnan(y)) and np.nanmax(np.abs(x - y)) < 1e-10


@pytest.mark.parametrize("trend", [0.0, 6.0, -6.0, 0.3])
@pytest.mark.parametrize("Lq,g,d,fp8", RANGES)
def test_blocks_with_many_tiles(Lq, g, d, fp8, trend):
    # scores that rise by `trend` a tile (6: the base moves with every tile, and only the last ones count), fall, or do neither
    K, V, table, scales, scale, Q, lens, rows = batch(Lq, g, d, fp8, trend, seed=Lq + d)
    w_in = torch.rand(B, 2, table.shape[1] * PAGE, generator=torch.Generator().manual_seed(1)).cuda()
    w = torch.full_like(w_in, 7.0)
    O = torch.full((B, Lq, 2 * g, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, 2 * g, Lq), 7.0, device="cuda")
    run(Q, K, V, table, scales, lens, rows, weights=w_in, weights_out=w, out=O, lse=lse)
    sa.poll_status()
    want = decode64(Q, K, V, table, lens, rows, S, T, MASK, PAGE, scale)
    ref.check_decode(O, lse, want, rows, d, fp8=fp8, w_in=w_in, w_out=w, kv_len=lens)
    for b in range(B):
        assert (O[b, rows[b]:] == 7.0).all() and (lse[b, :, rows[b]:] == 7.0).all() and (w[b, :, lens[b] if rows[b] else 0:] == 7.0).all()
    O2, l2 = run(Q, K, V, table, scales, lens, rows, out=torch.full_like(O, 7.0), lse=torch.full_like(lse, 7.0))
    assert torch.equal(O, O2) and torch.equal(lse, l2)


@pytest.mark.parametrize("trend", [0.0, 3.0])
@pytest.mark.parametrize("Lq,g,d,fp8", [c for c in RANGES if c[0] > 2])
def test_what_the_border_hides_in_the_middle_of_a_range(Lq, g, d, fp8, trend):
    # slots 768 to 1791 are seen by a local head's rows of the old segment, not by those of the new one: NaN keys and values that
    # are not finite there must leave the new rows' bits alone, and the old rows' other elements right
    K, V, table, scales, scale, Q, lens, rows = batch(Lq, g, d, fp8, trend, seed=Lq)
    rows = [Lq if b % 16 else 0 for b in range(B)]
    lens = [2048 + 1 + b % (Lq - 1) for b in range(B)]      # at least one row on each side of the border
    clean, lse = run(Q, K, V, table, scales, lens, rows, out=torch.zeros(B, Lq, 2 * g, d, dtype=torch.bfloat16, device="cuda"),
                     lse=torch.zeros(B, 2 * g, Lq, device="cuda"))
    hidden = [800, 831, 1000, 1001, 1063, 1290, 1500, 1700, 1790]
    put = lambda x, s, j, val, e=slice(None): x.view(torch.uint8 if fp8 else torch.bfloat16).__setitem__((table[s, j // PAGE].long(), j % PAGE, 0, e), val)
    nan = 0x7f if fp8 else math.nan
    Vi = V.clone()
    for s in range(12):
        for i, j in enumerate(hidden):
            put(Vi, s, j, nan if fp8 or i % 3 == 0 else math.inf if i % 3 == 1 else -math.inf, 3 + i)     # element 3 + i of one value row
    O, l2 = run(Q, K, Vi, table, scales, lens, rows, out=torch.zeros_like(clean), lse=torch.zeros_like(lse))
    sa.poll_status()
    assert torch.equal(l2, lse)
    assert torch.equal(O[:, :, g:], clean[:, :, g:])        # the other KV head
    old = torch.tensor([[lens[b] - Lq + t < 2048 for t in range(Lq)] for b in range(B)])
    there = torch.tensor([r > 0 for r in rows])[:, None].expand(B, Lq)
    new_rows, old_rows = (there & ~old).cuda(), (there & old).cuda()
    assert new_rows.any() and old_rows.any()
    assert torch.equal(O[new_rows], clean[new_rows])
    spoiled = torch.zeros(d, dtype=torch.bool)
    spoiled[3:3 + len(hidden)] = True
    got, base = O[old_rows][:, :g].float().cpu(), clean[old_rows][:, :g].float().cpu()
    assert not torch.isfinite(got[..., spoiled]).any()
    # the other elements: the same sum, taken in another order where a value row was added by itself, its weight rounded or not
    some = [b for b in range(B) if rows[b] > 0][:24]
    want = decode64(Q[some], K, V, table[some], [lens[b] for b in some], [Lq] * len(some), S, T, MASK, PAGE, scale)
    Of, keep = O[some].float().cpu().double().numpy()[..., (~spoiled).numpy()], (~spoiled).numpy()
    es = (d + 8) * ref.FP32 * want[3] + 2.0 ** -18
    bound = ((ref.FP16 if fp8 else ref.BF16) + 2 * es.transpose(0, 2, 1)[..., None]) * want[2][..., keep] + 1.02 * ref.BF16 * np.abs(want[0][..., keep])
    assert (np.abs(Of - want[0][..., keep]) <= bound).all()
    # keys too: every row that does not see them keeps its bits
    Kn = K.clone()
    for s in range(12):
        for j in hidden:
            put(Kn, s, j, nan)
    O, l2 = run(Q, Kn, Vi, table, scales, lens, rows, out=torch.zeros_like(clean), lse=torch.zeros_like(lse))
    sa.poll_status()
    assert torch.equal(O[new_rows], clean[new_rows]) and torch.equal(l2.transpose(1, 2)[new_rows], lse.transpose(1, 2)[new_rows])
    assert torch.isnan(O[old_rows][:, :g].float()).all() and torch.equal(O[:, :, g:], clean[:, :, g:])


# ---- eviction ---------------------------------------------------------------------------------------------------------

def choice(w, n, sink, recent, heavy):
    """ref.evict_choice for long sequences."""
    if n <= sink + recent + heavy:
        return np.arange(n)
    mid = w[sink:n - recent]
    j = np.arange(sink, n - recent)
    order = np.lexsort((j, -np.where(np.isnan(mid), 0, mid), np.isnan(mid)))
    return np.concatenate([np.arange(sink), np.sort(j[order[:heavy]]), np.arange(n - recent, n)])


# batch, KV heads, lengths (in turn), sink, recent, heavy: one block a head and more keys than fit beside sequences of fewer; two
# blocks a head that both read their keys again; two of which one does
LONG = [(16, 8, [60000, 41743, 41742, 300], 5, 777, 4001), (8, 8, [131072, 100001, 2500], 16, 1024, 3000), (8, 8, [82932, 82950], 3, 999, 20000)]


@pytest.mark.parametrize("kind", ["plain", "ties", "flat", "odd"])
@pytest.mark.parametrize("case", LONG, ids=lambda c: "b%d_h%d_n%d" % (c[0], c[1], c[2][0]))
def test_evictions_with_more_keys_than_a_block_keeps(case, kind):
    from test_gpu_paged import make_weights
    nb, Hkv, lens, sink, recent, heavy = case
    lens = [lens[b % len(lens)] for b in range(nb)]
    d, page, budget = 64, 256, sink + recent + heavy
    per, src = -(-budget // page), -(-max(lens) // page)
    g = torch.Generator().manual_seed(nb)
    K = torch.randint(-32768, 32767, (src + nb * per, page, Hkv, d), generator=g, dtype=torch.int16).cuda()     # bits, moved as they are
    V = torch.randint(-32768, 32767, K.shape, generator=g, dtype=torch.int16).cuda()
    K0, V0 = K.clone(), V.clone()
    order = torch.randperm(src + nb * per, generator=g).int()
    table, dst = order[:src].expand(nb, src).contiguous().cuda(), order[src:].reshape(nb, per).cuda()      # all read the same pages
    W = src * page
    w = make_weights(kind, nb, Hkv, W, seed=5).cuda()
    idx, n2, s2, w2 = sa.kv_evict(w, K.view(torch.bfloat16), V.view(torch.bfloat16), table, torch.tensor(lens, dtype=torch.int32, device="cuda"), dst, sink,
                                  recent, heavy)
    sa.poll_status()
    wc, want_idx, want_w = w.cpu().numpy(), np.full((nb, Hkv, budget), -1), torch.zeros_like(w)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            keep = choice(wc[b, h], n, sink, recent, heavy)
            want_idx[b, h, :len(keep)] = keep
            at = torch.from_numpy(keep).cuda()
            want_w[b, h, :len(keep)] = w[b, h, at]
            r = torch.arange(len(keep), device="cuda")
            for x, x0 in ((K, K0), (V, V0)):
                moved, rows = x[dst[b, r // page].long(), r % page, h], x0[table[b, at // page].long(), at % page, h]
                assert torch.equal(moved, rows), (b, h)
        assert (int(n2[b]), int(s2[b])) == (min(n, budget), n - min(n, budget))
    assert np.array_equal(idx.cpu().numpy(), want_idx)
    assert torch.equal(w2.view(torch.int32), want_w.view(torch.int32))
    assert torch.equal(K[table[0].long()], K0[table[0].long()]) and torch.equal(V[table[0].long()], V0[table[0].long()])


def test_the_long_choice_is_the_reference_s():
    for kind in ("plain", "ties", "flat", "odd"):
        from test_gpu_paged import make_weights
        w = make_weights(kind, 1, 1, 700, seed=2)[0, 0]
        for n, sink, recent, heavy in ((700, 3, 40, 100), (500, 0, 0, 499), (90, 5, 30, 60), (600, 1, 1, 0)):
            assert choice(w.numpy(), n, sink, recent, heavy).tolist() == ref.evict_choice(w.tolist(), n, sink, recent, heavy)


def test_a_captured_loop_with_an_eviction_leaves_the_same_bits():
    # tokens appended and attended over, an eviction, more tokens: captured and replayed, the cache is bit by bit what the same calls
    # made one by one leave
    nb, Hq, Hkv, d, page, seg, tail = 2, 8, 2, 128, 16, 32, 8
    sink, recent, heavy = 1, seg + tail, 6
    table = sa.rope_table_scaled(300, 64)
    g = torch.Generator().manual_seed(17)
    steps = [[torch.randn(nb, 1, H, d, generator=g).bfloat16().cuda() for H in (Hkv, Hkv, Hq)] for _ in range(9)]

    def make():
        c = ref.Cache([60, 75], Hkv, d, page, seed=19, spare=12, max_pages=6)
        c.table[0, 4], c.table[1, 5] = c.spare[10], c.spare[11]
        bt2 = torch.full((nb, 6), -1, dtype=torch.int32)
        bt2[:, :5] = torch.tensor(c.spare[:10], dtype=torch.int32).reshape(nb, 5)
        return dict(K=c.K, V=c.V, bt=c.table.clone().cuda(), n=c.dev["kv_len"].clone(), shift=torch.zeros(nb, dtype=torch.int32, device="cuda"),
                    w=torch.zeros(nb, Hkv, 110, device="cuda"), w2=torch.zeros(nb, Hkv, 110, device="cuda"), bt2=bt2.cuda(),
                    new=[t.clone() for t in steps[0]])

    def token(x, bt, w):
        x["n"] += 1
        q = sa.kv_append(x["new"][0], x["new"][1], x["K"], x["V"], x[bt], x["n"], table=table, Q=x["new"][2], pos_shift=x["shift"])
        return sa.seg_attn_decode(q, x["K"], x["V"], x[bt], x["n"], seg, tail, [0, 1], pos_shift=x["shift"], weights=x[w], weights_out=x[w])

    def evict(x):
        return sa.kv_evict(x["w"], x["K"], x["V"], x["bt"], x["n"], x["bt2"][:, :5], sink, recent, heavy, pos_shift=x["shift"], weights_out=x["w2"],
                           kv_len_out=x["n"], pos_shift_out=x["shift"])

    one, rep = make(), make()
    graphs = []
    state = {k: v.clone() for k, v in rep.items() if torch.is_tensor(v)}
    for f in (lambda: token(rep, "bt", "w"), lambda: evict(rep), lambda: token(rep, "bt2", "w2")):
        f()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f()
        graphs.append(gr)
    for k, v in state.items():
        rep[k].copy_(v)
    for i, new in enumerate(steps):
        for x in (one, rep):
            for to, t in zip(x["new"], new):
                to.copy_(t)
        if i == 4:
            evict(one)
            graphs[1].replay()
        token(one, "bt" if i < 4 else "bt2", "w" if i < 4 else "w2")
        graphs[0 if i < 4 else 2].replay()
        for k in ("K", "V"):
            assert torch.equal(one[k].view(torch.int16), rep[k].view(torch.int16)), (i, k)
        for k in ("w", "w2"):
            assert torch.equal(one[k], rep[k]), (i, k)
        assert torch.equal(one["n"], rep["n"]) and torch.equal(one["shift"], rep["shift"])
    sa.poll_status()
    assert not torch.equal(one["K"].view(torch.int16), make()["K"].view(torch.int16)) and one["n"].tolist() == [sink + recent + heavy + 5] * 2
