"""Scales of blocks that no append writes: zero, negative, not finite, and small or large throughout, in the attention, the eviction and the
append itself, against the definition (a stored element x stands for x times its block's scale) in 64 bits."""
import math

import numpy as np
import pytest
import torch

import blocks_ref as br
import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def attend(Q, K, V, ks, vs, table, n, S, T, mask, page, idx=None, block=0, q_len=None):
    """O, LSE of a sequence's last q_len rows and the bounds of their errors; K, V: stored values, ks, vs: their scales by row, float64.

    With u = 2^-24, d + 3 roundings of a score's terms and a few more of its weight and the sum (2^-18 for all orders, as in
    paged_ref.check_decode); weights times scales are fp16 numbers (2^-11), the largest of them 2^12 at least, below whose normal range
    half a step is 2^-25: 2^-37 of the largest weight times scale for each stored value, a block of scale zero (or of one that is not finite) counting with the largest of
    the others at most.  The output is rounded to bf16: 2^-8 of it, and below its normal range half a step, 2^-134."""
    q_len, Hq, d = Q.shape
    g = Hq // K.shape[2]
    out = []
    for t in range(q_len):
        for h in range(Hq):
            kv = h // g
            j = br.visible(n, q_len, t, mask[kv], S, T, 0, None if idx is None else idx[t, kv], block)
            at = np.asarray(table)[j // page], j % page, kv
            k, v, sv = K[at] * ks[at][:, None], V[at], vs[at]
            s = d ** -0.5 * (k @ Q[t, h])
            terms = d ** -0.5 * (np.abs(k) @ np.abs(Q[t, h])).max()
            p = np.exp(s - s.max())
            lse = s.max() + math.log(p.sum())
            p /= p.sum()
            fine = np.isfinite(sv) & (sv != 0)
            most = np.abs(sv[fine]).max() if fine.any() else 0.0
            with np.errstate(invalid="ignore"):
                O = p @ (v * sv[:, None])
            w = p * np.where(fine, np.abs(sv), most)
            es = (d + 8) * ref.FP32 * terms + 2.0 ** -18
            spread = p[fine] @ np.abs(v[fine] * sv[fine, None]) if fine.any() else np.zeros(d)
            stray = 2.0 ** -37 * w.max() * np.abs(v[fine]).sum(0)
            out.append((O, lse, (ref.FP16 + 2 * es) * spread + stray + 1.02 * ref.BF16 * np.abs(O) + 2.0 ** -134, es + 4 * ref.FP32 * abs(lse)))
    shape = lambda k, *s: np.array([x[k] for x in out]).reshape(q_len, Hq, *s)
    return shape(0, d), shape(1), shape(2, d), shape(3)


def compare(c, Q, S, T, mask, idx=None, block=0):
    """The attention over cache c against the definition; rows whose definition is not finite are not finite."""
    kw = {} if idx is None else dict(blocks=torch.from_numpy(idx).cuda(), block=block)
    O, lse = sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, **c.dev, **c.scales, **kw)
    sa.poll_status()
    K, V = (x.float().cpu().double().numpy() for x in (c.K, c.V))
    ks, vs = (br.by_row(c.scales[x], c.page) for x in ("k_scale", "v_scale"))
    for b, n in enumerate(c.lens):
        want = attend(Q[b].float().cpu().double().numpy(), K, V, ks, vs, c.table[b].numpy(), n, S, T, mask, c.page, None if idx is None else idx[b], block)
        o, l = O[b].float().cpu().double().numpy(), lse[b].T.cpu().double().numpy()
        assert (np.abs(l - want[1]) <= want[3]).all(), ("lse", b, float(np.nanmax(np.abs(l - want[1]))))
        fine = np.isfinite(want[0])
        assert np.array_equal(np.isfinite(o), fine), b
        err = np.abs(o - want[0])[fine]
        assert (err <= want[2][fine]).all(), ("O", b, float((err / want[2][fine]).max()))
    return O, lse


def put(c, b, blocks, value, head=slice(None), which="v_scale"):
    """This value for the scales of some blocks of sequence b."""
    per = c.page // c.rows
    for j in blocks:
        c.scales[which][int(c.table[b, j // per]), j % per, head] = value


def query(*shape, seed=0, size=1.0):
    return (size * torch.randn(*shape, generator=torch.Generator().manual_seed(50 + seed))).bfloat16().cuda()


# Lq, Hq: up to 8, 16, 32 and 64 rows to a KV head
ROWS = [(1, 4), (1, 24), (5, 8), (12, 8)]


@pytest.mark.parametrize("Lq,Hq", ROWS)
@pytest.mark.parametrize("d,page,rows", [(64, 32, 16), (128, 64, 64)])
@pytest.mark.parametrize("where", ["first", "middle", "last", "most", "every"])
def test_scales_of_zero(where, d, page, rows, Lq, Hq):
    lens = [700, 330, rows + 1]
    for e in (0, -110, 100):
        c = br.ScaledCache(lens, 2, d, page, rows, seed=d + Lq)
        c.scales["v_scale"].mul_(2.0 ** e)
        for b, n in enumerate(lens):
            m = -(-n // rows)
            put(c, b, dict(first=[0], middle=[m // 2], last=[m - 1], most=[j for j in range(m) if j != m * 2 // 3], every=range(m))[where], 0.0)
        O, _ = compare(c, query(3, Lq, Hq, d), 1 << 30, 0, [1, 1])
        assert where != "every" or not O.any()
        compare(c, query(3, Lq, Hq, d, seed=1), 64, 16, [1, 0])


@pytest.mark.parametrize("Lq,Hq", ROWS)
@pytest.mark.parametrize("e", [-140, -126, -122, -115, -110, 110, 119])
def test_scales_that_are_all_small_or_large(e, Lq, Hq):
    c = br.ScaledCache([900, 311], 2, 64, 64, 16, seed=3)
    c.scales["v_scale"].fill_(2.0 ** e)
    compare(c, query(2, Lq, Hq, 64), 1 << 30, 0, [1, 1])
    for b in range(2):      # and no powers of two, 2^30 apart
        put(c, b, range(0, c.lens[b] // 16, 3), 2.0 ** e * 1.5)
        put(c, b, range(1, c.lens[b] // 16, 3), 2.0 ** (e + 30 if e < 0 else e - 30) * 1.25)
    compare(c, query(2, Lq, Hq, 64, seed=1), 1 << 30, 0, [1, 1])


@pytest.mark.parametrize("e", [-126, -100, 0, 110])
@pytest.mark.parametrize("B", [1, 20])
def test_many_equal_scores_under_small_scales(B, e):
    # 128K slots of the same weight: their sum is 2^17 times a weight, whatever the scale
    n, page, d, Hkv = 131072, 256, 64, 2
    g = torch.Generator().manual_seed(1)
    V = (torch.randint(1, 9, (n // page, page, Hkv, d), generator=g).float() / 8).to(E4M3).cuda()
    K = torch.zeros(n // page, page, Hkv, d, device="cuda").to(E4M3)
    s = torch.full((n // page, page // 64, Hkv), 2.0 ** e, device="cuda")
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    O, lse = sa.seg_attn_decode(query(B, 1, 4, d), K, V, table, torch.full((B,), n, dtype=torch.int32, device="cuda"), 1 << 30, 0, [1] * Hkv,
                                k_scale=torch.ones_like(s), v_scale=s)
    sa.poll_status()
    mean = V.cpu().double().mean((0, 1)).repeat_interleave(2, 0) * 2.0 ** e      # [Hq, d]; values alike, so that every rounding is relative
    bound = (ref.FP16 + 1.02 * ref.BF16 + 2.0 ** -17) * mean + 2.0 ** -134
    assert ((O.cpu().double()[:, 0] - mean).abs() <= bound).all()
    assert ((lse.cpu().double() - math.log(n)).abs() <= 2.0 ** -18 + 4 * ref.FP32 * math.log(n)).all()


@pytest.mark.parametrize("Lq,Hq", ROWS)
def test_negative_scales(Lq, Hq):
    lens = [500, 130]
    c = br.ScaledCache(lens, 2, 128, 32, 16, seed=6, powers=False)
    for b, n in enumerate(lens):
        for j in range(0, -(-n // 16), 3):
            for x in ("k_scale", "v_scale"):
                put(c, b, [j + (x == "k_scale")] if j * 16 + 16 < n else [j], -0.3, which=x)
    compare(c, query(2, Lq, Hq, 128), 1 << 30, 0, [1, 1])
    compare(c, query(2, Lq, Hq, 128, seed=1), 64, 16, [1, 0])


@pytest.mark.parametrize("Lq,Hq", ROWS)
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_scales_that_are_not_finite(odd, Lq, Hq):
    # rows that see the block are not finite, in any dim; the LSE, and rows that do not see it, are what they are without it
    lens, S, T, rows = [400, 207], 48, 16, 16
    for blocks in ([0], [3], [10, 11]):
        c = br.ScaledCache(lens, 2, 64, 32, rows, seed=7)
        for b in range(2):
            put(c, b, blocks, odd, head=0)
        O, _ = compare(c, query(2, Lq, Hq, 64), S, T, [1, 0])
        assert not torch.isfinite(O[:, :, :Hq // 2].float()).any() and torch.isfinite(O[:, :, Hq // 2:].float()).all()
    # the new rows' own segment begins inside a tile: some of them see a block of the one before it, some do not
    c = br.ScaledCache([400 - 400 % S + Lq // 2 + 1], 1, 64, 32, rows, seed=8)
    put(c, 0, [(400 - 400 % S) // rows - 1], odd)
    compare(c, query(1, Lq, Hq, 64, seed=2), S, T, [2])
    compare(c, query(1, Lq, Hq, 64, seed=2), S, T, [0])


@pytest.mark.parametrize("kind", ["zero", "small", "negative", "nan"])
@pytest.mark.parametrize("d,Lq,Hq", [(64, 1, 4), (128, 3, 8), (64, 1, 24)])
def test_odd_scales_among_chosen_blocks(d, Lq, Hq, kind):
    lens, S, T, block, n, rows = [900, 400], 64, 16, 32, 6, 16
    c = br.ScaledCache(lens, 2, d, 64, rows, seed=9)
    idx = np.full((2, Lq, 2, n), -1, np.int32)
    idx[0, :, :, :5], idx[1, :, :, :3] = [0, 2, 5, 9, 17], [1, 3, 4]
    if kind == "small":
        c.scales["v_scale"].mul_(2.0 ** -115)
    for b, blocks in enumerate(([0, 1, 5, 18], [2, 3, 9])):      # 16-row blocks 0, 1: the first chosen one of the first sequence
        if kind != "small":
            put(c, b, blocks, dict(zero=0.0, negative=-1.5, nan=math.nan)[kind], head=slice(0, 1 if kind == "nan" else 2))
    compare(c, query(2, Lq, Hq, d), S, T, [1, 1], idx, block)


def test_scales_that_drift_along_parts_of_a_long_sequence():
    # parts of a row come from many thread blocks, whose scales are 2^98 apart from one end to the other, up and down, some of them zero
    n, page, d, rows = 20000, 64, 64, 64
    for up in (True, False):
        for seed in range(2):
            c = br.ScaledCache([n, n // 3], 2, d, page, rows, seed=seed)
            for b, m in enumerate(c.lens):
                k = -(-m // rows)
                for j in range(k):
                    at = j if up else k - 1 - j
                    put(c, b, [j], 0.0 if j % 7 == 2 or (seed and j < 40) else 2.0 ** (98 * at // (k - 1) - 49) * (1.0 if seed else 1.375))
            compare(c, query(2, 1, 4, d, seed=seed, size=0.3), 1 << 30, 0, [1, 1])


@pytest.mark.parametrize("unit", [1.0, 2.0 ** -70, 2.0 ** 80])
@pytest.mark.parametrize("d,page,rows", [(64, 32, 16), (128, 64, 64)])
def test_evicted_rows_keep_values_of_any_scale(d, page, rows, unit):
    # the new block's scale is the largest magnitude of its rows' finite ones; what a row stood for, it stands for afterwards
    n, Hkv, sink, recent, heavy = 300, 2, 3, 40, 50
    budget = sink + recent + heavy
    need = -(-budget // page)
    c = br.ScaledCache([n], Hkv, d, page, rows, seed=d, spare=3 + need)
    c.K.copy_((4 * torch.randn(c.K.shape, generator=torch.Generator().manual_seed(2))).clamp(-400, 400).cuda().to(E4M3))
    c.V.copy_((4 * torch.randn(c.K.shape, generator=torch.Generator().manual_seed(3))).clamp(-400, 400).cuda().to(E4M3))
    for x, shift in (("k_scale", 0), ("v_scale", 1)):
        for j in range(-(-n // rows)):
            put(c, 0, [j], unit * (0.5, -4.0, 0.0, -0.25, math.nan, 2.0)[(j + shift) % 6], which=x)
    dst = torch.tensor(c.spare[:need], dtype=torch.int32).view(1, need)
    W = c.max_pages * page
    w = torch.rand(1, Hkv, max(W, budget), generator=torch.Generator().manual_seed(1)).cuda()
    before = [x.cpu().clone() for x in (c.K, c.V, c.scales["k_scale"], c.scales["v_scale"])]
    idx, *_ = sa.kv_evict(w, c.K, c.V, dst_table=dst.cuda(), sink=sink, recent=recent, heavy=heavy, **c.dev, **c.scales)
    sa.poll_status()
    for x, s, pages, scales in ((0, 2, c.K, c.scales["k_scale"]), (1, 3, c.V, c.scales["v_scale"])):
        for h in range(Hkv):
            keep = idx[0, h].tolist()
            for r0 in range(0, budget, rows):
                at = [(int(c.table[0, j // page]), j % page) for j in keep[r0:r0 + rows]]
                src = torch.stack([before[s][p, q // rows, h] for p, q in at])
                fine = src[torch.isfinite(src)].abs()
                top = (fine.max().item() if len(fine) else 0.0) or 2.0 ** -40
                to, first = int(dst[0, r0 // page]), r0 % page
                assert scales[to, first // rows, h].item() == top
                want = torch.stack([before[x][p, q, h].float() for p, q in at]) * (src / top)[:, None]
                got = pages[to, first:first + len(at), h].cpu()
                same = lambda a: torch.where(br.bits(a) & 0x7f == 0x7f, 0x7f, br.bits(a))
                assert torch.equal(same(got), same(want.to(E4M3)))


@pytest.mark.parametrize("old", [-0.5, -64.0, 0.0, 3.0, 2.0 ** -60, -(2.0 ** 100), math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d,rows", [(64, 16), (128, 64)])
def test_rows_appended_to_a_block_of_any_scale(d, rows, old):
    # what the rows there stood for, they stand for afterwards: they are brought to the larger magnitude of the old scale and the new rows'
    n, Hkv, page = rows + rows // 2 + 3, 2, 2 * rows
    c = br.ScaledCache([n], Hkv, d, page, rows, seed=d)
    pages = [(4 * torch.randn(c.K.shape, generator=torch.Generator().manual_seed(k))).clamp(-400, 400).to(E4M3) for k in (1, 2)]
    c.K.copy_(pages[0].cuda()), c.V.copy_(pages[1].cuda())
    for x in ("k_scale", "v_scale"):
        put(c, 0, [0, 1], old, which=x)
    for Lq in (1, rows // 2):
        K, V = query(1, Lq, Hkv, d, seed=Lq, size=3.0), query(1, Lq, Hkv, d, seed=Lq + 1, size=100.0)
        before = [x.cpu().clone() for x in (c.K, c.V, c.scales["k_scale"], c.scales["v_scale"])]
        sa.kv_append(K, V, c.K, c.V, **c.dev, **c.scales)
        sa.poll_status()
        at = int(c.table[0, 0])
        for new, was, s0, stored, scales in ((K, before[0], before[2], c.K, c.scales["k_scale"]), (V, before[1], before[3], c.V, c.scales["v_scale"])):
            first = n - Lq
            for h in range(Hkv):
                x = new[0, :, h].float().cpu()
                s = s0[at, 1, h].item()
                want = max(br.scale_of(x.abs().max().item()), abs(s) if math.isfinite(s) else 0.0)
                assert scales[at, 1, h].item() == want
                there = (was[at, rows:first, h].float() * (torch.tensor(s) / want)).clamp(-448, 448)
                fresh = (x * (1 / torch.tensor(want))).clamp(-448, 448)
                same = lambda a: torch.where(br.bits(a) & 0x7f == 0x7f, 0x7f, br.bits(a))
                assert torch.equal(same(stored[at, rows:first, h].cpu()), same(there.to(E4M3)))
                assert torch.equal(same(stored[at, first:n, h].cpu()), same(fresh.to(E4M3)))
                assert torch.equal(br.bits(stored)[at, :rows, h].cpu(), br.bits(was)[at, :rows, h])
