"""Pages from requested lengths, 8-bit caches with a scale for each block, means of blocks, their choice and the attention over them, on
the GPU against references in whole numbers and 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

import blocks_ref as br
import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def ints(x, kind=torch.int32):
    return torch.tensor(x, dtype=kind, device="cuda")


def rand(*shape, seed=0, pad=0):
    """bf16 normal values, a slice of a wider tensor in the heads' dimension where `pad` says so."""
    g = torch.Generator().manual_seed(1000 + seed)
    return torch.randn(*shape[:2], shape[2] + pad, *shape[3:], generator=g).bfloat16().cuda()[:, :, :shape[2]]


def f64(t):
    return t.float().cpu().double().numpy()


def same8(got, want):
    """The same 8-bit values; a NaN's sign says nothing."""
    a, b = (torch.where(x & 0x7f == 0x7f, 0x7f, x) for x in (br.bits(got).cpu(), br.bits(want).cpu()))
    return torch.equal(a, b)


def refused():
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 1


# ---- pages ------------------------------------------------------------------------------------------------------------

def pool(B, page, per, n_pages, seed, most=None):
    """Sequences with pages of their own, and the list of the others."""
    r = random.Random(seed)
    order = list(range(n_pages))
    r.shuffle(order)
    lens, table = [], []
    for b in range(B):
        n = min(r.choice([0, 1, r.randint(0, most or per * page)]), len(order) * page)
        k = -(-n // page)
        table.append([order.pop() for _ in range(k)] + [-1] * (per - k))
        lens.append(n)
    return lens, table, order


def device_pool(lens, table, free, n_pages):
    return ints(lens), ints(table).reshape(len(lens), -1), ints(free + [-1] * (n_pages - len(free))), ints([len(free)])


@pytest.mark.parametrize("B,page,per,n_pages,Lq", [(1, 16, 4, 4, 1), (5, 16, 8, 30, 1), (64, 16, 40, 1500, 1), (64, 1, 60, 2000, 7), (33, 100, 9, 200, 300),
                                                   (300, 7, 5, 1200, 20), (1500, 16, 6, 6000, 3), (3000, 8, 4, 9000, 1), (40, 64, 40, 900, 2000),
                                                   (7, 48, 1, 7, 48), (2, 8, 3000, 4000, 20000)])
def test_resize_matches_the_definition(B, page, per, n_pages, Lq):
    for seed in range(3):
        r = random.Random(100 * seed + B)
        lens, table, free = pool(B, page, per, n_pages, seed, most=per * page if seed else per * page // 2)
        want = [r.choice([n, 0, max(0, n - r.randint(0, 2 * page)), min(per * page, n + r.randint(0, Lq)), min(per * page, n + Lq)]) for n in lens]
        shift = [r.randint(0, 9) for _ in lens] if seed == 1 else None
        n, t, f, c = device_pool(lens, table, free, n_pages)
        got = sa.pages_resize(ints(want), t, n, f, c, page, Lq, pos_shift=None if shift is None else ints(shift))
        sa.poll_status()
        T, N, F, q, slots, pos = br.resize(want, table, lens, free, len(free), page, Lq, shift)
        assert got[0].tolist() == N and got[1].item() == len(F) and got[2].tolist() == q
        assert got[3].tolist() == slots and got[4].tolist() == pos
        assert f[:len(F)].tolist() == F
        for b in range(B):
            k = -(-N[b] // page)
            assert t[b, :k].tolist() == T[b][:k]
        assert n.tolist() == lens and c.item() == len(free)      # the inputs are as they were


def test_resize_in_place_over_many_steps():
    # admission, growth, rolled-back tokens and ends, with the lengths and the list in place; no page is lost or held twice
    B, page, per, n_pages = 24, 8, 20, 60
    lens, table, free = [0] * B, [[-1] * per for _ in range(B)], list(range(n_pages))
    n, t, f, c = device_pool(lens, table, free, n_pages)
    r = random.Random(5)
    wide = torch.full((B, per + 3), -1, dtype=torch.int32, device="cuda")      # the table as a slice
    wide[:, :per] = t
    t = wide[:, :per]
    waited = 0
    for step in range(60):
        want = [r.choice([x + 1, x + 1, x + 1, min(x + 37, per * page), max(0, x - 3), 0]) if x + 1 < per * page else 0 for x in lens]
        sa.pages_resize(ints(want), t, n, f, c, page, 40, kv_len_out=n, free_count_out=c)
        table, lens, free, *_ = br.resize(want, table, lens, free, len(free), page, 40)
        waited += sum(a != b for a, b in zip(want, lens))
        assert n.tolist() == lens and c.item() == len(free) and f[:len(free)].tolist() == free
    sa.poll_status()
    assert waited > 20 and (wide[:, per:] == -1).all()
    held = [x for b in range(B) for x in t[b, :-(-lens[b] // page)].tolist()] + free
    assert sorted(held) == list(range(n_pages))


@pytest.mark.parametrize("Lq", [4, 3000])
def test_resize_refuses_numbers_out_of_range(Lq):
    # each stays as it is, the others go on; both sizes of call
    page, per, n_pages = 16, 400, 900
    lens, table, free = [40, 33, 20, 7], [[k * 3 + i for i in range(3)] + [-1] * (per - 3) for k in range(4)], list(range(20, 700))
    for want, bad in (([-1, 34, 21, 8], 0), ([per * page + 1, 34, 21, 8], 0), ([41, 33 + Lq + 1, 21, 8], 1)):
        n, t, f, c = device_pool(lens, table, free, n_pages)
        got = sa.pages_resize(ints(want), t, n, f, c, page, Lq)
        refused()
        fine = [l if b == bad else w for b, (w, l) in enumerate(zip(want, lens))]
        T, N, F, q, slots, pos = br.resize(fine, table, lens, free, len(free), page, Lq)
        assert got[0].tolist() == N and got[1].item() == len(F) and got[2].tolist() == q and got[3].tolist() == slots
    for wrong in (-1, per * page + 1, 1 << 30, -(1 << 31)):
        n, t, f, c = device_pool([wrong] + lens[1:], table, free, n_pages)
        got = sa.pages_resize(ints([50, 34, 21, 8]), t, n, f, c, page, Lq)
        refused()
        assert got[0].tolist() == [wrong, 34, 21, 8] and got[2].tolist() == [0, 1, 1, 1] and (got[3][0] == -1).all()
    # numbers of pages
    n, t, f, c = device_pool(lens, table, free[:-2] + [n_pages, -5], n_pages)
    got = sa.pages_resize(ints([50, 49, 21, 8]), t, n, f, c, page, 17 if Lq < 17 else Lq)
    refused()
    assert got[0].tolist() == [50, 49, 21, 8] and t[0, 3].item() == -1 and t[1, 3].item() == -1 and (got[3][0, 8:] == -1).all() and (got[3][0, :8] >= 0).all()
    for count in (-3, n_pages + 1):
        n, t, f, c = device_pool(lens, table, free, n_pages)
        got = sa.pages_resize(ints([41, 34, 21, 8]), t, n, f, ints([count]), page, Lq)
        refused()
        assert got[0].tolist() == [41, 34, 21, 8] and got[1].item() == (0 if count < 0 else n_pages)
    # more pages given back than the list has room for
    n, t, f, c = device_pool(lens, table, list(range(n_pages - 2)), n_pages)
    guard = f.clone()
    got = sa.pages_resize(ints([0, 33, 20, 7]), t, n, f, c, page, Lq)
    refused()
    assert got[1].item() == n_pages and f[n_pages - 2:].tolist() == table[0][:2] and torch.equal(f[:n_pages - 2], guard[:n_pages - 2])
    n, t, f, c = device_pool(lens, table, free, n_pages)
    got = sa.pages_resize(ints([41, 34, 21, 8]), t, n, f, c, page, Lq, pos_shift=ints([-1, 2, 0, 0]))
    refused()
    assert got[4][:2, 0].tolist() == [40, 35]
    sa.poll_status()


def test_resize_writes_the_lengths_where_they_were_asked_for():
    B, page, per, n_pages = 1500, 16, 6, 5000
    lens, table, free = pool(B, page, per, n_pages, 1)
    r = random.Random(2)
    want = [r.choice([0, x, min(per * page, x + 9)]) for x in lens]
    n, t, f, c = device_pool(lens, table, free, n_pages)
    w = ints(want)
    got = sa.pages_resize(w, t, n, f, c, page, 9, kv_len_out=w, free_count_out=c)
    sa.poll_status()
    T, N, F, q, slots, pos = br.resize(want, table, lens, free, len(free), page, 9)
    assert got[0] is w and w.tolist() == N and c.item() == len(F) and got[2].tolist() == q and got[3].tolist() == slots


def test_resize_without_pages_or_sequences():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    got = sa.pages_resize(ints([3, 0]), torch.empty(2, 0, dtype=torch.int32, device="cuda"), ints([0, 0]), e, ints([0]), 16, 4)
    refused()      # 3 rows are past a table without entries
    assert got[0].tolist() == [0, 0] and got[2].tolist() == [0, 0]
    got = sa.pages_resize(e, torch.empty(0, 4, dtype=torch.int32, device="cuda"), e, ints([1, 2]), ints([2]), 16, 4)
    assert got[0].numel() == 0
    got = sa.pages_resize(ints([20]), ints([[5, -1]]), ints([16]), ints([1, 2] + [-1] * 4), ints([2]), 16, 0)      # no room to grow in the call
    refused()
    assert got[0].tolist() == [16] and got[3].shape == (1, 0)
    sa.poll_status()


# ---- append ------------------------------------------------------------------------------------------------------------

APPEND = [
    # lens (after), Lq, q_len, Hq, Hkv, d, page, rows, rot, layout
    ([1], 1, None, 2, 1, 64, 16, 16, 64, "half"),
    ([20, 33, 17], 1, None, 4, 2, 128, 32, 16, 128, "half"),
    ([5, 33, 20], 5, [5, 0, 3], 8, 2, 128, 48, 16, 128, "interleaved"),
    ([300, 260], 256, None, 6, 3, 128, 64, 64, 32, "half"),
    ([100, 17], 17, [9, 17], 4, 4, 64, 96, 32, 48, "interleaved"),
    ([40], 40, None, 0, 2, 128, 16, 16, 96, "half"),                 # keys alone
    ([90, 65], 8, None, 0, 2, 64, 128, 128, 0, "half"),              # no rotation
    ([700, 500, 2], 500, [500, 500, 2], 16, 4, 128, 256, 128, 64, "interleaved"),
    ([131, 64, 129], 3, None, 4, 2, 128, 64, 64, 128, "half"),       # into half-filled blocks, across their border
    ([200], 150, None, 2, 2, 64, 128, 64, 16, "half"),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "n%d_q%d_d%d_p%d_b%d_r%d" % (max(c[0]), c[1], c[5], c[6], c[7], c[8]))
def test_append_finds_the_scales(case):
    lens, Lq, q_len, Hq, Hkv, d, page, rows, rot, layout = case
    B = len(lens)
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=lens[0])
    g = torch.Generator().manual_seed(77)
    size = torch.exp2(torch.randint(-6, 7, (B, Lq, 1, 1), generator=g).float())      # scales that grow, and stay
    mk = lambda H: (torch.randn(B, Lq, H + 1, d, generator=g) * size).bfloat16().cuda()[:, :, :H]
    Kn, Vn = mk(Hkv), mk(Hkv)
    Vn[0, 0, 0, :3] = torch.tensor([math.inf, math.nan, -math.inf])      # saturates, stays NaN, and has no say in the scale
    if Lq > 4:
        Kn[0, 3], Vn[0, 4] = 0, 0
    Q = mk(Hq) if Hq else None
    new = [Lq] * B if q_len is None else q_len
    shift = [3 * b for b in range(B)]
    table = sa.rope_table_scaled(max(lens) + 3 * B, rot) if rot else None
    want = [x.cpu().clone() for x in (c.K, c.V, c.scales["k_scale"], c.scales["v_scale"])]
    for b in range(B):
        first = lens[b] - new[b]
        k, v = Kn[b, :new[b]].float().cpu(), Vn[b, :new[b]].float().cpu()
        if rot:      # every product and sum rounded to 32 bits, as the kernel documents: the same bits
            k = torch.from_numpy(ref.rotate(k.numpy(), table[first + shift[b]:lens[b] + shift[b]].cpu().numpy(), layout)) if new[b] else k
        br.append(want[0], want[2], rows, k, first, lens[b], c.table[b].tolist(), page)
        br.append(want[1], want[3], rows, v, first, lens[b], c.table[b].tolist(), page)
    qo = torch.full_like(Q, 7.0) if Hq else None
    kw = dict(table=table, layout=layout, Q=Q, q_out=qo, pos_shift=ints(shift), q_len=None if q_len is None else ints(q_len), **c.dev, **c.scales)
    sa.kv_append(Kn, Vn, c.K, c.V, **kw)
    sa.poll_status()
    for got, w in zip((c.K, c.V), want):
        assert same8(got, w)
    for x, w in zip(("k_scale", "v_scale"), want[2:]):
        assert torch.equal(torch.nan_to_num(c.scales[x].cpu(), nan=-1.0), torch.nan_to_num(w, nan=-1.0))
    for b in range(B):
        if Hq:
            for t in range(new[b]):
                tab = table[lens[b] - new[b] + t + shift[b]].cpu().numpy()
                assert torch.equal(qo[b, t].cpu(), torch.from_numpy(ref.rotate(Q[b, t].float().cpu().numpy(), tab, layout)).bfloat16())
            assert (qo[b, new[b]:] == 7.0).all()
    # a call again changes nothing
    sa.kv_append(Kn, Vn, c.K, c.V, **kw)
    sa.poll_status()
    for got, w in zip((c.K, c.V), want):
        assert same8(got, w)


@pytest.mark.parametrize("d,rows", [(64, 16), (128, 64)])
def test_tokens_one_by_one_come_to_the_scales_of_all_at_once(d, rows):
    # the scales are those of one call; a value is off by one more rounding, at its own scale, where a scale grew after it
    n, Hkv, page = 150, 3, 2 * rows
    g = torch.Generator().manual_seed(4)
    size = torch.exp2(torch.arange(n).float() % 11 - 5)[:, None, None]
    K, V = ((torch.randn(1, n, Hkv, d, generator=g) * size).bfloat16().cuda() for _ in range(2))
    one, all_ = (br.ScaledCache([n], Hkv, d, page, rows, seed=1) for _ in range(2))
    sa.kv_append(K, V, all_.K, all_.V, **all_.dev, **all_.scales)
    for t in range(n):
        one.dev["kv_len"].fill_(t + 1)
        sa.kv_append(K[:, t:t + 1], V[:, t:t + 1], one.K, one.V, **one.dev, **one.scales)
    sa.poll_status()
    for x in ("k_scale", "v_scale"):
        assert torch.equal(torch.nan_to_num(one.scales[x]), torch.nan_to_num(all_.scales[x]))
    j = np.arange(n)
    for (a, b), x in zip(zip(one.values(), all_.values()), (K, V)):
        at = np.asarray(one.table[0])[j // page], j % page
        scale = f64(one.scales["k_scale" if x is K else "v_scale"])[at[0], at[1] // rows][..., None]
        true = f64(x)[0]
        step = np.maximum(2.0 ** -4 * np.abs(true), 2.0 ** -10 * scale)      # half a step of e4m3; of its lowest octave
        assert (np.abs(b[at] - true) <= step).all()
        assert (np.abs(a[at] - true) <= step + 2.0 ** -10 * scale).all()      # what was rounded first has whole steps above that octave


def test_append_leaves_out_rows_without_a_place():
    page, rows, Hkv, d = 32, 16, 2, 64
    table = sa.rope_table_scaled(60, d)
    for what in ("long", "negative", "short", "q_len", "shift", "position", "page"):
        c = br.ScaledCache([64, 40], Hkv, d, page, rows, seed=3)
        before = [x.clone() for x in (c.K, c.V, *c.scales.values())]
        Kn, Vn = rand(2, 5, Hkv, d, seed=1), rand(2, 5, Hkv, d, seed=2)
        lens, q, shift, kw = [64, 40], [5, 5], [0, 0], {}
        if what == "long":
            lens[0] = 66      # two rows past the table of 64
        if what == "negative":
            lens[0] = -1
        if what == "short":
            lens[0] = 3       # two rows in front of the first slot
        if what == "q_len":
            q[0] = 6
        if what == "shift":
            shift[0], kw = -1, dict(table=table)
        if what == "position":
            lens, kw = [64, 30], dict(table=table)      # positions 60.. are not there
        tab = c.table.clone()
        if what == "page":
            tab[0, 1] = c.K.shape[0]
        sa.kv_append(Kn, Vn, c.K, c.V, tab.cuda(), ints(lens), q_len=ints(q), pos_shift=ints(shift), **kw, **c.scales)
        refused()
        spared = dict(long=(59 + 2, 64), short=(0, 3), position=(59, 60)).get(what)
        changed = (br.bits(c.K) != br.bits(before[0])).any(-1).any(-1).cpu()
        rows_of = lambda b, lo, hi: {(int(tab[b, j // page]), j % page) for j in range(lo, hi)}
        allowed = rows_of(1, lens[1] - 5, lens[1]) | (rows_of(0, *spared) if spared else set())
        # blocks that had rows may have been brought to a larger scale
        allowed |= rows_of(1, (lens[1] - 5) // rows * rows, lens[1] - 5) | (rows_of(0, spared[0] // rows * rows, spared[0]) if spared else set())
        assert {tuple(x) for x in changed.nonzero().tolist()} <= allowed, what
        assert changed[tab[1, (lens[1] - 1) // page].long(), (lens[1] - 1) % page]      # the other sequence's rows are there
        if spared:
            assert changed[int(tab[0, (spared[1] - 1) // page]), (spared[1] - 1) % page]
    sa.poll_status()


# ---- attention over scales of blocks --------------------------------------------------------------------------------------

def check(O, lse, want, rows, d, fp8, w_in=None, w_out=None, kv_len=None):
    ref.check_decode(O, lse, want, rows, d, fp8=fp8, w_in=w_in, w_out=w_out, kv_len=kv_len)


DECODE = [
    # lens, Lq, q_len, Hq, Hkv, d, page, rows, S, T, mask
    ([1], 1, None, 1, 1, 64, 16, 16, 64, 16, [0]),
    ([0, 1, 2], 1, [0, 1, 1], 4, 2, 128, 16, 16, 64, 16, [1, 0]),
    ([517], 1, None, 32, 8, 128, 16, 16, 128, 32, [0, 0, 1, 0, 0, 2, 1, 0]),
    ([5, 700, 64, 65, 63, 129], 1, None, 8, 2, 128, 64, 32, 100, 37, [1, 0]),
    ([333, 80], 1, None, 3, 3, 64, 48, 16, 50, 50, [2, 1, 0]),
    ([300, 41, 7, 130], 5, [5, 0, 3, 5], 8, 2, 128, 32, 32, 32, 8, [0, 1]),
    ([260, 3], 4, [4, 3], 20, 1, 64, 128, 128, 64, 64, [1]),
    ([150], 33, None, 8, 4, 128, 48, 16, 40, 10, [0, 1, 2, 0]),
    ([2, 5], 5, None, 4, 2, 128, 16, 16, 16, 4, [0, 1]),
    ([5000, 1200], 1, None, 16, 2, 128, 64, 64, 1 << 30, 0, [1, 0]),
    ([9000, 17], 2, None, 64, 8, 128, 256, 128, 4096, 1024, [1] * 8),
    ([4097], 1, None, 8, 1, 64, 128, 64, 2048, 512, [1]),
    ([400, 90], 70, [70, 33], 4, 1, 128, 64, 64, 128, 32, [0]),
    ([300, 41], 40, [40, 0], 8, 2, 64, 16, 16, 100, 20, [1, 2]),
    ([(37 * b) % 211 for b in range(300)], 1, [1 if (37 * b) % 211 and b % 7 else 0 for b in range(300)], 4, 2, 64, 16, 16, 50, 20, [0, 1]),
]


def run_scaled(c, Q, S, T, mask, q_len=None, shift=None, want_w=False, **kw):
    B, Lq, Hq, d = Q.shape
    rows, cap = [Lq] * B if q_len is None else list(q_len), c.max_pages * c.page
    O, lse = torch.full((B, Lq, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq, Lq), 7.0, device="cuda")
    w = torch.full((B, c.K.shape[2], cap), 7.0, device="cuda") if want_w else None
    sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, q_len=None if q_len is None else ints(q_len),
                       pos_shift=None if shift is None else ints(shift), out=O, lse=lse, weights_out=w, **c.dev, **c.scales, **kw)
    sa.poll_status()
    want = br.attend(f64(Q), *c.values(), c.table.numpy(), c.lens, rows, S, T, mask, d ** -0.5, c.page, shift=shift, cap=cap,
                     v_scale=br.by_row(c.scales["v_scale"], c.page))
    check(O, lse, want, rows, d, True, w_out=w, kv_len=c.lens)
    for b in range(B):
        assert (O[b, rows[b]:] == 7.0).all() and (lse[b, :, rows[b]:] == 7.0).all()
        if w is not None:
            assert (w[b, :, (c.lens[b] if rows[b] else 0):] == 7.0).all()
    return O, lse


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "n%s_q%d_h%d_%d_d%d_p%d_b%d" % (max(c[0]), c[1], c[3], c[4], c[5], c[6], c[7]))
def test_decode_with_scales_matches_the_definition(case, powers):
    lens, Lq, q_len, Hq, Hkv, d, page, rows, S, T, mask = case
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=len(lens) + lens[-1], powers=powers)
    Q = rand(len(lens), Lq, Hq, d)
    a = run_scaled(c, Q, S, T, mask, q_len=q_len, want_w=True)
    b = run_scaled(c, Q, S, T, mask, q_len=q_len)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d,Lq", [(64, 1), (128, 1), (128, 4), (64, 12), (128, 40)])
def test_scales_far_apart(d, Lq):
    # scales of V over 60 powers of two, and of K over 12: a weight's share of the output goes by its scale, its share of the sum does not
    lens, Hkv, page, rows = [900, 311], 2, 64, 16
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=d + Lq)
    g = torch.Generator().manual_seed(9)
    for x, span in (("k_scale", 6), ("v_scale", 30)):
        s = torch.exp2(torch.randint(-span, span + 1, c.scales[x].shape, generator=g).float()).cuda()
        s[torch.isnan(c.scales[x])] = math.nan
        c.scales[x].copy_(s)
    run_scaled(c, 0.05 * rand(2, Lq, 4, d), 64, 16, [1, 0])
    c.scales["v_scale"].fill_(2.0 ** -100)
    run_scaled(c, 0.05 * rand(2, Lq, 4, d), 1 << 30, 0, [1, 1])
    c.scales["v_scale"].fill_(2.0 ** 100)
    run_scaled(c, 0.05 * rand(2, Lq, 4, d), 1 << 30, 0, [1, 1])


@pytest.mark.parametrize("e", [-30, 3])
@pytest.mark.parametrize("Hq", [4, 16, 64])
def test_scores_too_large_for_a_fraction(Hq, e):
    # scores of 2e9, whose fp32 steps are 128: a base is rounded by more than the room above it, and nothing may overflow for it
    n, d, page = 300, 64, 16
    c = br.ScaledCache([n], 1, d, page, 16, seed=2)
    br.bits(c.K)[:] = br.bits(torch.full((1,), 1.0).to(E4M3)).item()
    for j, x in ((7, 448.0), (130, 448.0), (131, 416.0)):
        c.K[c.table[0, j // page].long(), j % page] = torch.full((1, d), x, device="cuda").to(E4M3)
    c.scales["k_scale"].fill_(8.0)
    c.scales["v_scale"].fill_(2.0 ** e)
    Q = torch.full((1, 1, Hq, d), 65536.0, dtype=torch.bfloat16, device="cuda")
    O, lse = sa.seg_attn_decode(Q, c.K, c.V, S=1 << 30, T=0, head_past_mask=[1], **c.dev, **c.scales)
    sa.poll_status()
    # which of the two equal keys wins is within the scores' rounding; the row is their mean with some weights
    vals = ref.rows_of(c.V, c.table[0].numpy(), n, page)[[7, 130], 0] * 2.0 ** e
    slack = (2 * ref.FP16 + 1.02 * ref.BF16) * np.abs(vals).max(0)
    got = f64(O)[0, 0]
    assert (got >= vals.min(0) - slack).all() and (got <= vals.max(0) + slack).all()
    top = d * 65536.0 * 448 * 8 * d ** -0.5
    assert (np.abs(lse.cpu().double().numpy() - top) <= 8 * ref.FP32 * top).all()


def test_two_streams_at_once():
    # the same calls on two streams with buffers of their own, and a captured step replayed beside them
    lens, S, T, block, n, page = [3000, 2000, 900], 64, 16, 16, 8, 64
    c = br.ScaledCache(lens, 2, 128, page, 16, seed=2)
    Qs = [rand(3, 2, 16, 128, seed=k) for k in range(3)]
    outs = [old_means(c, block) for _ in range(3)]

    def step(k):
        sa.blocks_summarise(c.K, c.dev["block_table"], c.dev["kv_len"], 3000, *outs[k], k_scale=c.scales["k_scale"])
        idx = sa.blocks_select(Qs[k], *outs[k], c.dev["block_table"], c.dev["kv_len"], page, S, T, n, head_past_mask=[1, 1])
        return (idx,) + sa.seg_attn_decode(Qs[k], c.K, c.V, S=S, T=T, head_past_mask=[1, 1], blocks=idx, block=block, **c.dev, **c.scales)
    want = [[x.clone() for x in step(k)] for k in range(3)]
    torch.cuda.synchronize()
    streams, gr = [torch.cuda.Stream() for _ in range(3)], torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=streams[2]):
        kept = step(2)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(25):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(step(k))
        with torch.cuda.stream(streams[2]):
            gr.replay()
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for x in got[k] for a, b in zip(x, want[k]))
    assert all(torch.equal(a, b) for a, b in zip(kept, want[2]))
    sa.poll_status()


@pytest.mark.parametrize("e", [-38, -20, 0, 25])
def test_the_lse_does_not_lose_what_the_scales_of_v_are_away(e):
    # scores near zero, so that the LSE is near ln n; a sum over 2^e in fp32 would be off by 2^-18 and more of it
    for n, parts in ((1, False), (3, False), (700, True)):
        c = br.ScaledCache([n] * 2, 2, 64, 16, 16, seed=n)
        for x, s in (("k_scale", 2.0 ** -12), ("v_scale", 2.0 ** e)):
            c.scales[x].fill_(s)
        Q = rand(2, 1, 4, 64)
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, S=1 << 30, T=0, head_past_mask=[1, 1], **c.dev, **c.scales)
        sa.poll_status()
        want = br.attend(f64(Q), *c.values(), c.table.numpy(), c.lens, [1, 1], 1 << 30, 0, [1, 1], 64 ** -0.5, 16)
        # a score's error, and a few roundings of numbers below log2 n + 1: of the sum, its logarithm and the conversion
        bound = (64 + 8) * ref.FP32 * want[3] + 16 * ref.FP32 * (math.log(n) + 1)
        assert (np.abs(lse.cpu().double().numpy() - want[1]) <= bound).all()


def test_small_weights_beside_a_dominant_key():
    # 32K slots of which the first takes all but a thousandth of the weight and has no value: what comes out is the small weights' work.
    # Its own block's scale is the largest of all, or the smallest.
    n, B, Hkv, g, page, d, tail = 32768, 64, 4, 4, 256, 128, 0.001
    for top in (2.0 ** -2, 2.0 ** -30, 2.0 ** 6):
        gen = torch.Generator().manual_seed(3)
        k, v = 4 * torch.randn(n // page, page, Hkv, d, generator=gen), 4 * torch.randn(n // page, page, Hkv, d, generator=gen) + 4
        ks, vs = torch.full((n // page, page // 64, Hkv), 0.25), torch.full((n // page, page // 64, Hkv), 0.25)
        Q = torch.randn(B, 1, Hkv * g, d, generator=gen)
        k[..., 0], k[0, 0], v[0, :64] = 0, 0, 0      # the first block has no values at all
        Q[..., 0], k[0, 0, :, 0] = 4.0, (math.log(n / tail) + 0.5) * d ** 0.5
        vs[0, 0] = top
        K, V, Q = k.to(E4M3).cuda(), v.to(E4M3).cuda(), Q.bfloat16()
        table = torch.arange(n // page, dtype=torch.int32).expand(B, -1).contiguous()
        O, lse = sa.seg_attn_decode(Q.cuda(), K, V, table.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"), 1 << 30, 0, [1] * Hkv,
                                    k_scale=ks.cuda(), v_scale=vs.cuda())
        sa.poll_status()
        some = [0, 63]
        Kd, Vd = br.dequantised(K, ks), br.dequantised(V, vs)
        Or, lr, spread, terms, _ = br.attend(f64(Q[some]), Kd, Vd, table[some].numpy(), [n] * 2, [1] * 2, 1 << 30, 0, [1] * Hkv, d ** -0.5, page)
        # as in check_decode; a number below fp16's normal range is off by half a step of it, 2^-25, where the largest weight times its
        # scale is 2^12 at least: the first key's, of weight 1, where its scale is large, else that of the small ones
        es = (d + 8) * ref.FP32 * terms + 2.0 ** -18
        size = np.abs(ref.rows_of(V, table[0].numpy(), n, page)).sum(0).repeat(g, 0)      # [Hq, d], in units of the scales
        bound = (ref.FP16 + 2 * es.transpose(0, 2, 1)[..., None]) * spread + 1.02 * ref.BF16 * np.abs(Or) + 2.0 ** -37 * max(top, 0.25) * size
        err = np.abs(f64(O[some]) - Or)
        assert (err <= bound).all(), (top, float((err / bound).max()))
        assert (np.abs(lse[some].cpu().double().numpy() - lr) <= es + 4 * ref.FP32 * np.abs(lr)).all()


@pytest.mark.parametrize("Lq,Hq,d", [(6, 4, 128), (6, 12, 64), (20, 4, 128), (40, 4, 64)])
def test_rows_nobody_sees_do_not_matter(Lq, Hq, d):
    lens, Hkv, page, rows, S, T = [Lq + 64, Lq + 31], 2, 32, 16, 32, 8
    mask = [0, 1]
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=5)
    Q = rand(2, Lq, Hq, d)
    clean, lse = run_scaled(c, Q, S, T, mask)
    last = Lq - 2
    for fill in (0x7f, 0xff):
        K, V = c.K.clone(), c.V.clone()
        for b, n in enumerate(lens):
            for j in range(n - Lq + last, n):
                br.bits(K)[c.table[b, j // page].long(), j % page] = fill
                br.bits(V)[c.table[b, j // page].long(), j % page] = fill
            low = min(ref.lowest_visible(n - Lq + t, S, T, 0, 0) for t in range(Lq))
            for j in range(0, low):
                br.bits(K)[c.table[b, j // page].long(), j % page, 0] = fill
                br.bits(V)[c.table[b, j // page].long(), j % page, 0] = fill
        O, l2 = sa.seg_attn_decode(Q, K, V, S=S, T=T, head_past_mask=mask, **c.dev, **c.scales)
        sa.poll_status()
        assert torch.equal(O[:, :last], clean[:, :last]) and torch.equal(l2[:, :, :last], lse[:, :, :last])
        assert not torch.isfinite(O[:, last:].float()).all()
        # a cached V that is not finite reaches those that see it, scaled
        O, l2 = sa.seg_attn_decode(Q, c.K, V, S=S, T=T, head_past_mask=mask, **c.dev, **c.scales)
        assert torch.equal(l2, lse) and torch.equal(O[:, :last], clean[:, :last]) and not torch.isfinite(O[:, last:].float()).any()


# ---- eviction ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,page,rows,lens,sink,recent,heavy", [(64, 16, 16, [200, 10, 40], 2, 20, 18), (128, 64, 32, [500, 131], 0, 64, 33), (128, 128, 128, [700], 4, 100, 200),
                                                               (64, 96, 32, [300, 299], 1, 0, 98), (128, 32, 16, [90], 0, 45, 0)])
def test_evicted_rows_keep_their_values(d, page, rows, lens, sink, recent, heavy):
    B, Hkv, budget = len(lens), 3, sink + recent + heavy
    need = -(-budget // page)
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=d, spread=5, spare=3 + B * need)
    dst = torch.tensor(c.spare[:B * need], dtype=torch.int32).view(B, need)
    W = c.max_pages * page
    w = torch.rand(B, Hkv, max(W, budget), generator=torch.Generator().manual_seed(1)).cuda()
    old = [x.cpu().clone() for x in (c.K, c.V, c.scales["k_scale"], c.scales["v_scale"])]
    idx, n2, s2, w2 = sa.kv_evict(w, c.K, c.V, dst_table=dst.cuda(), sink=sink, recent=recent, heavy=heavy, **c.dev, **c.scales)
    sa.poll_status()
    want = [x.clone() for x in old]
    for b, n in enumerate(lens):
        for h in range(Hkv):
            keep = ref.evict_choice(w[b, h].tolist(), n, sink, recent, heavy)
            assert idx[b, h].tolist() == keep + [-1] * (budget - len(keep))
            for x, s in ((0, 2), (1, 3)):
                for r0 in range(0, len(keep), rows):
                    at = [(int(c.table[b, j // page]), j % page) for j in keep[r0:r0 + rows]]
                    src = torch.stack([old[s][p, q // rows, h] for p, q in at])
                    to, first = int(dst[b, r0 // page]), r0 % page
                    want[s][to, first // rows, h] = src.max()
                    y = torch.stack([old[x][p, q, h].float() for p, q in at]) * (src / src.max())[:, None]
                    br.bits(want[x])[to, first:first + len(at), h] = br.bits(y.to(E4M3))
        assert n2[b].item() == min(n, budget) and s2[b].item() == n - min(n, budget)
    assert same8(c.K, want[0]) and same8(c.V, want[1])
    for x, y in (("k_scale", want[2]), ("v_scale", want[3])):
        assert torch.equal(torch.nan_to_num(c.scales[x].cpu(), nan=-1.0), torch.nan_to_num(y, nan=-1.0))
    # and the attention goes on over the compacted cache
    Q = rand(B, 1, 6, d)
    O, lse = sa.seg_attn_decode(Q, c.K, c.V, dst.cuda(), n2, 1 << 30, 0, [1] * Hkv, **c.scales)
    sa.poll_status()
    x = br.attend(f64(Q), *c.values(), dst.numpy(), n2.tolist(), [1] * B, 1 << 30, 0, [1] * Hkv, d ** -0.5, page, v_scale=br.by_row(c.scales["v_scale"], page))
    check(O, lse, x, [1] * B, d, True)
    bad = c.dev["block_table"].clone()
    bad[0, 0], d2 = -9, dst.clone()
    d2[-1, 0] = 1 << 20
    sa.kv_evict(w, c.K, c.V, bad, c.dev["kv_len"], d2.cuda(), sink, recent, heavy, **c.scales)
    refused()


# ---- layouts, empty caches, numbers out of range ------------------------------------------------------------------------------

def test_layouts_and_strides():
    lens, mask, S, T, block, n, page = [330, 147], [0, 1, 1, 1], 64, 16, 32, 3, 64
    for kind in ("bf16", "heads", "blocks"):      # pages by heads, queries as a slice, outputs of their own strides
        c = cache_of(kind, lens, 4, 64, page, block, seed=4, head_major=True)
        Q = rand(2, 3, 8, 64, pad=2)
        idx = random_choice(lens, [3, 3], 3, 4, S, T, block, n, seed=5)
        a = run_chosen(c, Q, S, T, mask, idx, block)
        wide = torch.full((2, c.max_pages + 5), -1, dtype=torch.int32, device="cuda")
        wide[:, :c.max_pages] = c.dev["block_table"]
        out = torch.zeros(2, 8, 3, 64, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        _, lse = sa.seg_attn_decode(Q, c.K, c.V, wide[:, :c.max_pages], c.dev["kv_len"], S, T, mask, blocks=torch.from_numpy(idx).cuda(), block=block, out=out,
                                    **c.scales)
        assert torch.equal(out, a[0]) and torch.equal(lse, a[1])
        sums, scale = old_means(c, block)
        sa.blocks_summarise(c.K, wide[:, :c.max_pages], c.dev["kv_len"], 400, sums, scale, k_scale=c.scales.get("k_scale"))
        X = br.dequantised(c.K, c.scales.get("k_scale"))
        got = sa.blocks_select(Q, sums, scale, wide[:, :c.max_pages], c.dev["kv_len"], page, S, T, n, head_past_mask=mask)
        for b, m in enumerate(lens):
            for k in range(m // block):
                at, row = int(c.table[b, k * block // page]), k * block % page
                mq, ms = br.means(X[at, row:row + block], block)
                assert np.array_equal(sums[at, row // block].cpu().numpy(), mq) and np.array_equal(scale[at, row // block].cpu().numpy(), ms)
            want = br.select(f64(Q[b]), sums.cpu().numpy(), scale.cpu().numpy(), c.table[b].tolist(), m, 3, S, T, mask, page, block, n, 0)
            assert np.array_equal(got[b].cpu().numpy(), want)
        if kind == "blocks":
            run_scaled(c, Q, S, T, mask, shift=[70, 0])
            new = rand(2, 5, 4, 64, seed=8), rand(2, 5, 4, 64, seed=9)
            flat = [x.contiguous() for x in (c.K, c.V, c.scales["k_scale"], c.scales["v_scale"])]
            sa.kv_append(*new, c.K, c.V, **c.dev, **c.scales)
            sa.kv_append(*new, flat[0], flat[1], k_scale=flat[2], v_scale=flat[3], **c.dev)
            assert same8(c.K, flat[0]) and same8(c.V, flat[1]) and torch.equal(torch.nan_to_num(c.scales["k_scale"]), torch.nan_to_num(flat[2]))
    sa.poll_status()


def test_caches_without_pages_and_rows_before_the_first_slot():
    e = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    z = ints([0, 0, 0])
    for Lq in (1, 2):
        idx = torch.full((3, Lq, 2, 4), -1, dtype=torch.int32, device="cuda")
        for kind in (torch.bfloat16, E4M3):
            K = torch.empty(0, 32, 2, 64, device="cuda").to(kind)
            s = {} if kind == torch.bfloat16 else dict(k_scale=torch.ones(0, 2, 2, device="cuda"), v_scale=torch.ones(0, 2, 2, device="cuda"))
            O, lse = sa.seg_attn_decode(rand(3, Lq, 4, 64), K, K, e, z, 64, 16, [0, 1], blocks=idx, block=16, **s)
            sa.poll_status()
            assert not O.any() and (lse == -math.inf).all()
            sa.blocks_summarise(K, e, z, 5, torch.empty(0, 2, 2, 64, dtype=torch.int8, device="cuda"), torch.empty(0, 2, 2, device="cuda"), k_scale=s.get("k_scale"))
            if s:
                O, lse = sa.seg_attn_decode(rand(3, Lq, 4, 64), K, K, e, z, 64, 16, [0, 1], **s)
                assert not O.any() and (lse == -math.inf).all()
            if s:      # rows without a place are reported, with queries and without
                for q in (None, rand(3, Lq, 4, 64)):
                    sa.kv_append(rand(3, Lq, 2, 64), rand(3, Lq, 2, 64), K, K, e, ints([1, 0, 2]), table=sa.rope_table_scaled(8, 64), Q=q, **s)
                    refused()
        got = sa.blocks_select(rand(3, Lq, 4, 64), torch.empty(0, 2, 2, 64, dtype=torch.int8, device="cuda"), torch.empty(0, 2, 2, device="cuda"), e, z, 32, 64, 16, 4,
                               head_past_mask=[1, 1])
        assert (got == -1).all()
    sa.poll_status()
    for kind in ("bf16", "blocks"):      # more new rows than slots: the first see nothing
        c = cache_of(kind, [2, 40], 1, 64, 32, 16, seed=1)
        idx = random_choice([2, 40], [4, 4], 4, 1, 8, 4, 16, 2, seed=1)
        O, lse = run_chosen(c, rand(2, 4, 2, 64), 8, 4, [1], idx, 16)
        assert not O[0, :2].any() and (lse[0, :, :2] == -math.inf).all()


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_numbers_out_of_range_are_reported_and_not_followed(kind):
    lens, S, T, block, n, page = [300, 200], 64, 16, 16, 4, 32
    c = cache_of(kind, lens, 2, 64, page, block, seed=9)
    idx = random_choice(lens, [1, 1], 1, 2, S, T, block, n, seed=2)
    Q, mask = rand(2, 1, 4, 64), [1, 0]
    clean, l0 = run_chosen(c, Q, S, T, mask, idx, block)
    sums, scale = (x.cuda() for x in random_means(c, block, 1))
    want = sa.blocks_select(Q, sums, scale, c.dev["block_table"], c.dev["kv_len"], page, S, T, n, head_past_mask=mask)
    full = c.table.clone().clamp(min=0).cuda()
    for bad_len, q in ((-1, 1), (c.max_pages * page + 1, 1), (300, -1), (300, 2)):
        kw = dict(q_len=ints([q, 1]))
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, full, ints([bad_len, 200]), S, T, mask, blocks=torch.from_numpy(idx).cuda(), block=block, **kw, **c.scales)
        refused()
        assert torch.equal(O[1], clean[1]) and torch.equal(lse[1], l0[1])
        got = sa.blocks_select(Q, sums, scale, full, ints([bad_len, 200]), page, S, T, n, head_past_mask=mask, **kw)
        refused()
        assert torch.equal(got[1], want[1])
        before = sums.clone()
        sa.blocks_summarise(c.K, full, ints([bad_len, 200]), 1, before, scale.clone(), k_scale=c.scales.get("k_scale"), **kw)
        refused()
        if kind == "blocks":
            O, lse = sa.seg_attn_decode(Q, c.K, c.V, full, ints([bad_len, 200]), S, T, mask, **kw, **c.scales)
            refused()
            a, b = sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, **c.dev, **c.scales)
            assert torch.equal(O[1], a[1]) and torch.equal(lse[1], b[1])
    sa.poll_status()


# ---- means of blocks --------------------------------------------------------------------------------------------------------

MEANS = [
    # lens, Lq, q_len, Hkv, d, page, block
    ([16], 1, None, 1, 64, 16, 16),
    ([15, 16, 17, 32], 1, None, 2, 128, 32, 16),
    ([300, 64, 63, 0], 70, [70, 64, 3, 0], 3, 128, 128, 64),
    ([700, 513], 700, [700, 513], 2, 64, 128, 128),
    ([200], 500, None, 2, 128, 96, 32),                      # all of it, and more asked for
]


def old_means(c, block):
    n_pages, _, Hkv, d = c.K.shape
    return torch.full((n_pages, c.page // block, Hkv, d), 9, dtype=torch.int8, device="cuda"), torch.full((n_pages, c.page // block, Hkv), 7.0, device="cuda")


@pytest.mark.parametrize("kind", ["bf16", "heads", "blocks"])
@pytest.mark.parametrize("case", MEANS, ids=lambda c: "n%d_q%d_d%d_p%d_b%d" % (max(c[0]), c[1], c[4], c[5], c[6]))
def test_means_match_the_definition(case, kind):
    lens, Lq, q_len, Hkv, d, page, block = case
    rows = 16 if block == 32 else block
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=Lq, powers=False) if kind == "blocks" else ref.Cache(lens, Hkv, d, page, fp8=kind == "heads", seed=Lq)
    sums, scale = old_means(c, block)
    want_q, want_s = sums.cpu().numpy().copy(), scale.cpu().numpy().copy()
    X = br.dequantised(c.K, c.scales.get("k_scale"))
    for b, n in enumerate(lens):
        new = Lq if q_len is None else q_len[b]
        for k in range(max(0, n - new) // block, n // block if new else 0):
            at, row = int(c.table[b, k * block // page]), k * block % page
            want_q[at, row // block], want_s[at, row // block] = br.means(X[at, row:row + block], block)
    sa.blocks_summarise(c.K, c.dev["block_table"], c.dev["kv_len"], Lq, sums, scale, q_len=None if q_len is None else ints(q_len),
                        k_scale=c.scales.get("k_scale"))
    sa.poll_status()
    assert np.array_equal(scale.cpu().numpy(), want_s) and np.array_equal(sums.cpu().numpy(), want_q)


def test_means_of_blocks_that_are_not_finite_or_all_zero():
    c = ref.Cache([64], 2, 64, 16, seed=1)
    c.K[c.table[0, 0].long(), 3, 0, 5] = math.inf
    c.K[c.table[0, 1].long(), 3, 1, 5] = math.nan
    c.K[c.table[0, 2].long()] = 0
    sums, scale = old_means(c, 16)
    sa.blocks_summarise(c.K, c.dev["block_table"], c.dev["kv_len"], 64, sums, scale)
    sa.poll_status()
    s, q = scale.cpu()[c.table[0].long(), 0], sums.cpu()[c.table[0].long(), 0]
    assert math.isnan(s[0, 0]) and math.isnan(s[1, 1]) and not (q[0, 0].any() or q[1, 1].any() or q[2].any()) and (s[2] == 0).all()
    assert torch.isfinite(s[[0, 1, 3, 3], [1, 0, 0, 1]]).all() and (q[[0, 1, 3, 3], [1, 0, 0, 1]].abs().amax(-1) == 127).all()
    bad = c.table.clone()
    bad[0, 1] = -7
    sa.blocks_summarise(c.K, bad.cuda(), c.dev["kv_len"], 64, sums, scale)
    refused()


# ---- the choice of blocks ---------------------------------------------------------------------------------------------------

SELECT = [
    # lens, Lq, q_len, Hq, Hkv, d, page, block, S, T, mask, n, sink
    ([500], 1, None, 4, 1, 64, 32, 16, 32, 8, [1], 4, 0),
    ([3000, 40, 0, 700], 1, [1, 1, 0, 1], 8, 4, 128, 64, 32, 100, 30, [1, 0, 1, 2], 7, 1),
    ([5000, 333], 5, [5, 2], 8, 2, 128, 48, 16, 64, 64, [1, 1], 64, 2),
    ([9000], 2, None, 64, 1, 64, 128, 64, 1000, 10, [1], 128, 0),
    ([20000, 19999, 64], 3, None, 6, 2, 128, 128, 128, 256, 256, [0, 1], 1, 1),
    ([8200], 1, None, 3, 3, 128, 16, 16, 16, 0, [1, 1, 1], 128, 128),
]


def random_means(c, block, seed):
    g = torch.Generator().manual_seed(seed)
    n_pages, _, Hkv, d = c.K.shape
    sums = torch.randint(-127, 128, (n_pages, c.page // block, Hkv, d), generator=g).to(torch.int8)
    return sums, torch.rand((n_pages, c.page // block, Hkv), generator=g)


@pytest.mark.parametrize("case", SELECT, ids=lambda c: "n%d_q%d_h%d_%d_d%d_b%d_n%d" % (max(c[0]), c[1], c[3], c[4], c[5], c[7], c[11]))
def test_selection_matches_the_definition(case):
    lens, Lq, q_len, Hq, Hkv, d, page, block, S, T, mask, n, sink = case
    B = len(lens)
    c = ref.Cache(lens, Hkv, 64, page, seed=n)
    c.K = torch.empty(c.K.shape[:3] + (d,), device="meta")
    new = [Lq] * B if q_len is None else q_len
    for kind in ("random", "coarse", "equal", "nan"):
        sums, scale = random_means(c, block, n)
        if kind == "coarse":      # many equal scores
            sums, scale = (sums // 100).to(torch.int8), torch.ones_like(scale)
        if kind == "equal":
            sums[:] = 1
            scale[:] = 0.5
        if kind == "nan":
            scale[torch.rand(scale.shape, generator=torch.Generator().manual_seed(1)) < 0.5] = math.nan
        Q = rand(B, Lq, Hq, d, seed=n, pad=2)
        out = torch.full((B, Lq, Hkv, n), 7, dtype=torch.int32, device="cuda")
        got = sa.blocks_select(Q, sums.cuda(), scale.cuda(), c.dev["block_table"], c.dev["kv_len"], page, S, T, n, sink=sink, head_past_mask=mask,
                               q_len=None if q_len is None else ints(q_len), out=out)
        sa.poll_status()
        assert got is out
        for b in range(B):
            want = br.select(f64(Q[b, :new[b]]), sums.numpy(), scale.numpy(), c.table[b].tolist(), lens[b], new[b], S, T, mask, page, block, n, sink)
            assert np.array_equal(got[b, :new[b]].cpu().numpy(), want), (kind, b)
            assert (got[b, new[b]:] == 7).all()


@pytest.mark.parametrize("lens,Hkv,block", [([140000], 1, 16), ([280000, 150001], 2, 16), ([600000], 1, 16)])
def test_selection_over_many_blocks(lens, Hkv, block):
    # slices for two, four and eight thread blocks
    page, n, S, T, d = 512, 50, 4096, 100, 64
    B = len(lens)
    per = max(-(-x // page) for x in lens)
    g = torch.Generator().manual_seed(2)
    table = torch.stack([torch.randperm(B * per, generator=g)[:per] for _ in range(B)]).int()
    for coarse in (False, True):
        sums = torch.randint(-127, 128, (B * per, page // block, Hkv, d), generator=g).to(torch.int8)
        scale = torch.rand((B * per, page // block, Hkv), generator=g) + 0.5
        if coarse:
            sums, scale = (sums // 120).to(torch.int8), torch.ones_like(scale)
        Q = rand(B, 1, 2 * Hkv, d, seed=1)
        got = sa.blocks_select(Q, sums.cuda(), scale.cuda(), table.cuda(), ints(lens), page, S, T, n, sink=3, head_past_mask=[1] * Hkv)
        sa.poll_status()
        for b in range(B):
            want = br.select(f64(Q[b]), sums.numpy(), scale.numpy(), table[b].tolist(), lens[b], 1, S, T, [1] * Hkv, page, block, n, 3)
            assert np.array_equal(got[b].cpu().numpy(), want), (coarse, b)


def test_selection_with_shifts_and_queries_that_are_not_finite():
    lens, page, block, S, T, n, Hkv, d = [900, 640], 32, 16, 64, 16, 5, 2, 64
    c = ref.Cache(lens, Hkv, d, page, seed=2)
    sums, scale = random_means(c, block, 3)
    Q = rand(2, 2, 4, d)
    Q[1, 0, 0, 3], Q[1, 1, 2] = math.inf, 0
    shift = [130, 0]
    got = sa.blocks_select(Q, sums.cuda(), scale.cuda(), c.dev["block_table"], c.dev["kv_len"], page, S, T, n, head_past_mask=[1, 1], pos_shift=ints(shift))
    sa.poll_status()
    for b in range(2):
        want = br.select(f64(Q[b]), sums.numpy(), scale.numpy(), c.table[b].tolist(), lens[b], 2, S, T, [1, 1], page, block, n, 0, shift=shift[b])
        assert np.array_equal(got[b].cpu().numpy(), want)
    assert got[1, 0, 0].tolist() == list(range(n))      # every score zero
    t = c.table.clone()
    t[0, 4] = 1 << 20      # its blocks rank lowest
    got = sa.blocks_select(Q, sums.cuda(), scale.cuda(), t.cuda(), c.dev["kv_len"], page, S, T, n, head_past_mask=[1, 1])
    refused()
    assert not ((got[0] == 8) | (got[0] == 9)).any()


# ---- attention over chosen blocks -------------------------------------------------------------------------------------------

ATTEND = [
    # lens, Lq, q_len, Hq, Hkv, d, page, block, S, T, mask, n
    ([500], 1, None, 1, 1, 64, 32, 16, 32, 8, [1], 4),
    ([3000, 40, 0, 700, 1], 1, [1, 1, 0, 1, 1], 8, 4, 128, 64, 32, 100, 30, [1, 0, 1, 2], 7),
    ([1500, 333], 5, [5, 2], 32, 2, 128, 48, 16, 64, 64, [1, 1], 64),
    ([2600], 2, None, 20, 1, 64, 128, 64, 1000, 10, [1], 128),
    ([4000, 3999, 64], 3, None, 6, 2, 128, 128, 128, 256, 256, [0, 1], 1),
    ([1200, 64], 2, [2, 1], 64, 8, 64, 16, 16, 16, 0, [1] * 8, 40),
    ([3, 30], 4, [3, 4], 4, 2, 128, 32, 32, 8, 8, [1, 2], 3),
    ([(53 * b) % 391 for b in range(150)], 1, [1 if (53 * b) % 391 and b % 5 else 0 for b in range(150)], 8, 2, 64, 32, 16, 40, 9, [1, 0], 6),
]


def random_choice(lens, new, Lq, Hkv, S, T, block, n, seed, shift=None):
    """Lists as a selection leaves them: ascending, then -1; of random lengths."""
    r = random.Random(seed)
    idx = np.full((len(lens), Lq, Hkv, n), -1, np.int32)
    for b, x in enumerate(lens):
        for t in range(new[b]):
            e, sh = x - new[b] + t, shift[b] if shift else 0
            room = br.first_whole(e + sh, S, T, sh, block) // block if e >= 0 else 0
            for h in range(Hkv):
                k = sorted(r.sample(range(room), min(room, r.choice([n, n, r.randint(0, n)]))))
                idx[b, t, h, :len(k)] = k
    return idx


def run_chosen(c, Q, S, T, mask, idx, block, q_len=None, shift=None, fine=True, **kw):
    B, Lq, Hq, d = Q.shape
    rows = [Lq] * B if q_len is None else list(q_len)
    O, lse = torch.full((B, Lq, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq, Lq), 7.0, device="cuda")
    sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, q_len=None if q_len is None else ints(q_len), out=O, lse=lse,
                       pos_shift=None if shift is None else ints(shift), blocks=torch.from_numpy(idx).cuda(), block=block, **c.dev, **c.scales, **kw)
    sa.poll_status() if fine else refused()
    vals = [br.dequantised(x, c.scales.get(s)) for x, s in ((c.K, "k_scale"), (c.V, "v_scale"))]
    want = br.attend(f64(Q), *vals, c.table.numpy(), c.lens, rows, S, T, mask, d ** -0.5, c.page, shift=shift, idx=idx, block=block,
                     v_scale=br.by_row(c.scales["v_scale"], c.page, len(c.K)) if c.scales else None)
    check(O, lse, want, rows, d, bool(c.scales))
    for b in range(B):
        assert (O[b, rows[b]:] == 7.0).all() and (lse[b, :, rows[b]:] == 7.0).all()
    return O, lse


def cache_of(kind, lens, Hkv, d, page, block, seed, **kw):
    rows = {16: 16, 32: 16, 64: 32, 128: 128}[block]
    return br.ScaledCache(lens, Hkv, d, page, rows, seed=seed, **kw) if kind == "blocks" else ref.Cache(lens, Hkv, d, page, fp8=kind == "heads", seed=seed, **kw)


@pytest.mark.parametrize("kind", ["bf16", "heads", "blocks"])
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "n%s_q%d_h%d_%d_d%d_p%d_b%d_n%d" % (max(c[0]), c[1], c[3], c[4], c[5], c[6], c[7], c[11]))
def test_attention_over_chosen_blocks_matches_the_definition(case, kind):
    lens, Lq, q_len, Hq, Hkv, d, page, block, S, T, mask, n = case
    c = cache_of(kind, lens, Hkv, d, page, block, seed=n)
    idx = random_choice(lens, [Lq] * len(lens) if q_len is None else q_len, Lq, Hkv, S, T, block, n, seed=n)
    Q = rand(len(lens), Lq, Hq, d)
    O, lse = run_chosen(c, Q, S, T, mask, idx, block, q_len=q_len)
    # every row by itself gives the same (to the order of a sum), and the queries' place may take the outputs
    q = Q.clone()
    O2, l2 = sa.seg_attn_decode(q, c.K, c.V, S=S, T=T, head_past_mask=mask, q_len=None if q_len is None else ints(q_len), out=q,
                                blocks=torch.from_numpy(idx).cuda(), block=block, **c.dev, **c.scales)
    for b in range(len(lens)):
        m = Lq if q_len is None else q_len[b]
        assert torch.equal(O[b, :m], O2[b, :m]) and torch.equal(lse[b, :, :m], l2[b, :, :m])


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_shifted_positions_and_a_choice(kind):
    lens, shift, S, T, block, n = [400, 260], [100, 0], 64, 16, 16, 6
    c = cache_of(kind, lens, 3, 64, 32, block, seed=6)
    idx = random_choice(lens, [2, 2], 2, 3, S, T, block, n, seed=1, shift=shift)
    run_chosen(c, rand(2, 2, 6, 64), S, T, [0, 1, 2], idx, block, shift=shift)


@pytest.mark.parametrize("kind", ["bf16", "heads", "blocks"])
def test_all_blocks_are_the_whole_past(kind):
    lens, S, T, block, page = [1000, 77, 300], 64, 16, 16, 64
    c = cache_of(kind, lens, 2, 128, page, block, seed=2)
    idx = np.full((3, 1, 2, 64), -1, np.int32)
    for b, x in enumerate(lens):
        room = br.first_whole(x - 1, S, T, 0, block) // block
        idx[b, :, :, :room] = np.arange(room)
    Q = rand(3, 1, 8, 128)
    a = run_chosen(c, Q, S, T, [1, 0], idx, block)
    b = sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=[1, 0], **c.dev, **c.scales)
    assert (a[1] - b[1]).abs().max() <= 1e-5 and (a[0].float() - b[0].float()).abs().max() <= 2 * ref.BF16 * b[0].float().abs().max()


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_lists_out_of_order_count_up_to_there(kind):
    lens, S, T, block, n = [800, 500], 64, 16, 16, 40
    c = cache_of(kind, lens, 1, 128, 32, block, seed=3)
    room = [br.first_whole(x - 1, S, T, 0, block) // block for x in lens]
    good = np.full((2, 1, 1, n), -1, np.int32)
    good[1, 0, 0, :3] = [1, 5, 9]
    for bad in ([3, 3], [3, 7, 5], [0, 2, room[0]], [room[0] + 1], [-2], [4, -1, 6], [1, 1 << 30], [5, -(1 << 31)], list(range(33)) + [32], list(range(39)) + [38]):
        idx = good.copy()
        idx[0, 0, 0, :len(bad)] = bad
        run_chosen(c, rand(2, 1, 4, 128), S, T, [1], idx, block, fine=bad == [4, -1, 6])
    sa.poll_status()


@pytest.mark.parametrize("kind", ["bf16", "heads", "blocks"])
def test_what_was_not_chosen_does_not_matter(kind):
    lens, S, T, block, n, page = [600, 410], 64, 16, 16, 5, 32
    c = cache_of(kind, lens, 2, 64, page, block, seed=4)
    idx = random_choice(lens, [1, 1], 1, 2, S, T, block, n, seed=3)
    Q = rand(2, 1, 6, 64)
    clean, lse = run_chosen(c, Q, S, T, [1, 1], idx, block)
    seen = {(b, h): set(br.visible(lens[b], 1, 0, 1, S, T, 0, idx[b, 0, h], block).tolist()) for b in range(2) for h in range(2)}
    for x in (c.K, c.V):
        for b, m in enumerate(lens):
            for j in range(m):
                for h in range(2):
                    if j not in seen[b, h]:
                        if kind == "bf16":
                            x[c.table[b, j // page].long(), j % page, h] = math.nan
                        else:
                            br.bits(x)[c.table[b, j // page].long(), j % page, h] = 0x7f
    O, l2 = sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=[1, 1], blocks=torch.from_numpy(idx).cuda(), block=block, **c.dev, **c.scales)
    sa.poll_status()
    assert torch.equal(O, clean) and torch.equal(lse, l2)
    t = c.table.clone()      # a chosen block on a page that is not there, and a kept one without a page of its own: not visible
    k = int(idx[0, 0, 0, 0])
    t[0, k * block // page] = 99999
    sa.seg_attn_decode(Q, c.K, c.V, t.cuda(), c.dev["kv_len"], S, T, [1, 1], blocks=torch.from_numpy(idx).cuda(), block=block, **c.scales)
    refused()


def test_no_weights_beside_a_choice():
    c = ref.Cache([100], 2, 64, 32, seed=1)
    idx = torch.full((1, 1, 2, 4), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(sa.SegAttnError):
        sa.seg_attn_decode(rand(1, 1, 4, 64), c.K, c.V, S=64, T=16, blocks=idx, block=16, weights_out=torch.zeros(1, 2, 128, device="cuda"), **c.dev)
    with pytest.raises(ValueError):
        sa.seg_attn_decode(rand(1, 1, 4, 64), c.K, c.V, S=64, T=16, blocks=idx[:, :, :1], block=16, **c.dev)


# ---- together ---------------------------------------------------------------------------------------------------------------

class Loop:
    """A decoding step of everything, on buffers of its own."""

    def __init__(self, B, Hq, Hkv, d, page, rows, block, n_pages, per, S, T, mask, n, fp8=True, seed=0):
        self.k = dict(page=page, S=S, T=T, mask=mask, n=n, block=block)
        z = lambda *s, kind=torch.float32: torch.zeros(s, dtype=kind, device="cuda")
        kind = E4M3 if fp8 else torch.bfloat16
        self.K, self.V = z(n_pages, page, Hkv, d).to(kind), z(n_pages, page, Hkv, d).to(kind)
        self.scales = dict(k_scale=z(n_pages, page // rows, Hkv), v_scale=z(n_pages, page // rows, Hkv)) if fp8 else {}
        self.sums, self.sum_scale = z(n_pages, page // block, Hkv, d, kind=torch.int8), z(n_pages, page // block, Hkv)
        self.table, self.n = torch.full((B, per), -1, dtype=torch.int32, device="cuda"), ints([0] * B)
        self.free, self.count = torch.arange(n_pages, dtype=torch.int32, device="cuda"), ints([n_pages])
        self.rope = sa.rope_table_scaled(per * page, d)

    def step(self, want, Q, Kn, Vn):
        k = self.k
        n, _, q_len, slots, pos = sa.pages_resize(want, self.table, self.n, self.free, self.count, k["page"], Q.shape[1], kv_len_out=self.n, free_count_out=self.count)
        kw = dict(block_table=self.table, kv_len=n, q_len=q_len)
        qr = sa.kv_append(Kn, Vn, self.K, self.V, table=self.rope, Q=Q, **kw, **self.scales)
        sa.blocks_summarise(self.K, self.table, n, Q.shape[1], self.sums, self.sum_scale, q_len=q_len, k_scale=self.scales.get("k_scale"))
        idx = sa.blocks_select(qr, self.sums, self.sum_scale, self.table, n, k["page"], k["S"], k["T"], k["n"], sink=1, head_past_mask=k["mask"], q_len=q_len)
        O, lse = sa.seg_attn_decode(qr, self.K, self.V, S=k["S"], T=k["T"], head_past_mask=k["mask"], blocks=idx, block=k["block"], **kw, **self.scales)
        return O, lse, idx, q_len, qr, slots, pos


@pytest.mark.parametrize("fp8", [True, False])
def test_a_loop_on_the_device(fp8):
    # prompts, tokens, a draft rolled back, ends and admissions: the steps are captured once for each width and replayed, and every
    # step's choice and attention is compared with the definition on what the cache then holds
    B, Hq, Hkv, d, page, rows, block, per, S, T, n = 4, 8, 2, 64, 32, 16, 16, 20, 48, 16, 4
    mask = [1, 0]
    lp = Loop(B, Hq, Hkv, d, page, rows, block, 70, per, S, T, mask, n, fp8=fp8)
    graphs = {}
    for Lq in (1, 3, 120):
        want, Q, Kn, Vn = ints([0] * B), rand(B, Lq, Hq, d), rand(B, Lq, Hkv, d, seed=1), rand(B, Lq, Hkv, d, seed=2)
        lp.step(want, Q, Kn, Vn)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = lp.step(want, Q, Kn, Vn)
        graphs[Lq] = gr, want, Q, Kn, Vn, out
    lens, r, seed = [0] * B, random.Random(3), 0
    for step in range(40):
        Lq = 120 if step in (0, 1, 2, 3, 20) else r.choice([1, 1, 3])
        ask = [x + (r.randint(1, 120) if Lq == 120 else r.choice([Lq, 1])) for x in lens]
        if step % 9 == 8:
            ask[r.randrange(B)] = 0
        if step % 7 == 5:
            b = r.randrange(B)
            ask[b] = max(0, lens[b] - 5)
        gr, want, Q, Kn, Vn, (O, lse, idx, q_len, qr, slots, pos) = graphs[Lq]
        seed += 1
        want.copy_(ints(ask))
        for x, s in ((Q, 0), (Kn, 1), (Vn, 2)):
            x.copy_(rand(*x.shape, seed=10 * seed + s))
        gr.replay()
        sa.poll_status()
        was, lens, q = lens, lp.n.tolist(), q_len.tolist()
        assert all(a == b or a == c for a, b, c in zip(lens, ask, was)) and q == [max(0, a - b) for a, b in zip(lens, was)]
        table = lp.table.cpu().numpy()
        held = [p for b in range(B) for p in table[b, :-(-lens[b] // page)].tolist()]
        assert sorted(held + lp.free[:lp.count.item()].tolist()) == list(range(70))
        K, V = br.dequantised(lp.K, lp.scales.get("k_scale")), br.dequantised(lp.V, lp.scales.get("v_scale"))
        flat = torch.from_numpy(K).reshape(-1, Hkv, d)
        for b in range(B):
            for t in range(q[b]):      # the slot map and the positions name the rows that the append wrote
                turned = ref.rotate(f64(Kn[b, t]), lp.rope[pos[b, t]].cpu().double().numpy(), "half")
                # half a step of what holds it; a row that a later one of the same block made coarser has one more, of the lowest octave
                top = np.abs(K[table[b][(was[b] + t) // page]]).max()
                bound = (2.0 ** -4 if fp8 else ref.BF16) * np.abs(turned) + (2.0 ** -16 * top + 1e-6 if fp8 else 1e-6)
                assert (np.abs(flat[slots[b, t]].numpy() - turned) <= bound).all()
            if q[b]:
                want_idx = br.select(f64(qr[b, :q[b]]), lp.sums.cpu().numpy(), lp.sum_scale.cpu().numpy(), table[b], lens[b], q[b], S, T, mask, page, block, n, 1)
                assert np.array_equal(idx[b, :q[b]].cpu().numpy(), want_idx)
                far = br.first_whole(lens[b] - 1, S, T, 0, block) // block
                for j in range(far):      # the means that can be chosen are those of the rows
                    at, row = table[b][j * block // page], j * block % page
                    mq, ms = br.means(K[at, row:row + block], block)
                    assert np.array_equal(lp.sums[at, row // block].cpu().numpy(), mq) and np.array_equal(lp.sum_scale[at, row // block].cpu().numpy(), ms)
        some = [q[b] if step % 4 == 0 or q[b] < 4 else 0 for b in range(B)]
        if any(some):
            x = br.attend(f64(qr), K, V, table, lens, q, S, T, mask, d ** -0.5, page, idx=idx.cpu().numpy(), block=block,
                          v_scale=br.by_row(lp.scales["v_scale"], page) if fp8 else None)
            check(O, lse, x, q, d, fp8)
    assert max(lens) > 250 and min(br.first_whole(max(lens) - 1, S, T, 0, block) // block, 99) > n


def test_calls_on_a_given_stream_allocate_there():
    lens, S, T, block, n, page = [3000, 2000], 64, 16, 16, 8, 64
    c = br.ScaledCache(lens, 2, 128, page, 16, seed=12)
    sums, scale = random_means(c, block, 1)
    sums, scale = sums.cuda(), scale.cuda()
    Q = rand(2, 1, 16, 128)
    lens_d, table, free, count = device_pool([30, 40], [[0, -1, -1], [1, -1, -1]], list(range(2, 40)), 40)

    def call(**kw):
        idx = sa.blocks_select(Q, sums, scale, c.dev["block_table"], c.dev["kv_len"], page, S, T, n, head_past_mask=[1, 1], **kw)
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=[1, 1], blocks=idx, block=block, **c.dev, **c.scales, **kw)
        return (idx, O, lse) + sa.pages_resize(ints([70, 41]), table, lens_d, free, count, 64, 50, **kw)
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(30):
        got.append(call(stream=side))
        torch.full((1 << 22,), math.nan, device="cuda")
    side.synchronize()
    torch.cuda.synchronize()
    for x in got:
        for a, b in zip(x, want):
            assert torch.equal(a, b)
    sa.poll_status()


@pytest.mark.parametrize("Lq,Hq", [(1, 4), (2, 20), (9, 4)])
def test_nothing_is_written_behind_the_workspaces(Lq, Hq):
    B, Hkv, d, page = 3, 2, 64, 32
    c = br.ScaledCache([64] * B, Hkv, d, page, 16, seed=1)
    idx = torch.full((B, Lq, Hkv, 3), -1, dtype=torch.int32, device="cuda")
    idx[..., 0] = 0
    (view, *_), sc = sa.paged._scaled_cache(c.K, c.V, c.dev["block_table"], c.dev["kv_len"], None, None, **c.scales)
    for choice in (None, sa.paged._CHOICE.pack(idx.data_ptr(), 3, 16)):
        need = sa.lib().seg_attn_decode_blocks_workspace_bytes(view, sc, choice, Lq, Hq, 0)
        buf = torch.full((need + (1 << 16),), 0x5a, dtype=torch.uint8, device="cuda")
        kw = {} if choice is None else dict(blocks=idx, block=16)
        sa.seg_attn_decode(rand(B, Lq, Hq, d), c.K, c.V, S=16, T=4, head_past_mask=[0, 1], workspace=buf[:need], **c.dev, **c.scales, **kw)
        sa.poll_status()
        assert (buf[need:] == 0x5a).all()
    need = sa.lib().seg_pages_workspace_bytes(5)
    buf = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    t = torch.arange(15, dtype=torch.int32, device="cuda").view(5, 3)
    for width in (2, 2000):
        sa.pages_resize(ints([33] * 5), t, ints([32] * 5), torch.arange(40, dtype=torch.int32, device="cuda"), ints([25]), 16, width, workspace=buf[:need])
        sa.poll_status()
        assert (buf[need:] == 0x5a).all()


def test_offsets_past_32_bits():
    page, Hkv, d = 32, 2, 128
    gap = (1 << 32) + 4096
    buf = torch.zeros(gap + page * Hkv * d, dtype=torch.uint8, device="cuda")
    K = buf.view(E4M3).as_strided((2, page, Hkv, d), (gap, Hkv * d, d, 1))
    wide = torch.zeros((1 << 31) + 64, device="cuda").as_strided((2, 2, Hkv), (1 << 31, 2, 1))
    c = br.ScaledCache([60], Hkv, d, page, 16, seed=3, spare=0)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    n, Kn, Vn = ints([60]), rand(1, 60, Hkv, d, seed=1), rand(1, 60, Hkv, d, seed=2)
    small_v = torch.zeros(2, 2, Hkv, device="cuda")
    kw = dict(block_table=table, kv_len=n)
    sa.kv_append(Kn, Vn, K, c.V, k_scale=wide, v_scale=small_v, **kw)
    sa.kv_append(Kn, Vn, c.K, c.V, k_scale=c.scales["k_scale"], v_scale=small_v, **kw)
    sa.poll_status()
    assert torch.equal(wide[1], c.scales["k_scale"][1]) and torch.equal(br.bits(K)[1], br.bits(c.K)[1]) and torch.equal(br.bits(K)[0, :28], br.bits(c.K)[0, :28])
    Q = rand(1, 1, 4, d)
    idx = ints([[[[0], [0]]]])
    a, b = (sa.seg_attn_decode(Q, k, c.V, S=8, T=4, head_past_mask=[1, 1], k_scale=s, v_scale=small_v, blocks=idx, block=16, **kw)
            for k, s in ((K, wide), (c.K, c.scales["k_scale"])))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    got = []
    for k, s in ((K, wide), (c.K, c.scales["k_scale"])):
        sums, scale = torch.zeros(2, 2, Hkv, d, dtype=torch.int8, device="cuda"), torch.zeros(2, 2, Hkv, device="cuda")
        sa.blocks_summarise(k, table, n, 60, sums, scale, k_scale=s)
        got.append((sums, scale))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    sa.poll_status()
