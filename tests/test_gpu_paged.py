"""The paged cache's operators on the GPU against 64-bit references: decoding attention, append, eviction."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu


def rand_q(B, Lq, Hq, d, seed=0, pad_heads=0):
    g = torch.Generator().manual_seed(1000 + seed)
    return torch.randn(B, Lq, Hq + pad_heads, d, generator=g).bfloat16().cuda()[:, :, :Hq]


def f64(t):
    return t.float().cpu().double().numpy()


def run_decode(c, Q, S, T, mask, q_len=None, shift=None, weights=None, want_weights=False, poll=True):
    B, Lq, Hq, d = Q.shape
    Hkv = c.K.shape[2]
    rows = [Lq] * B if q_len is None else list(q_len)
    dev = dict(q_len=None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda"),
               pos_shift=None if shift is None else torch.tensor(shift, dtype=torch.int32, device="cuda"))
    O = torch.full((B, Lq, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, Hq, Lq), 7.0, device="cuda")
    w = torch.full((B, Hkv, c.max_pages * c.page), 7.0, device="cuda") if want_weights else None
    sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, weights=weights, weights_out=w, out=O, lse=lse, **c.dev, **c.scales, **dev)
    if poll:
        sa.poll_status()
    want = ref.decode(f64(Q), c.K, c.V, c.table.numpy(), c.lens, rows, S, T, mask, d ** -0.5, c.page, shift=shift, **c.ref_scales())
    ref.check_decode(O, lse, want, rows, d, fp8=bool(c.scales), w_in=weights, w_out=w, kv_len=c.lens)
    for b in range(B):      # rows that are not there, and slots behind the end, are left as they were
        assert (O[b, rows[b]:] == 7.0).all() and (lse[b, :, rows[b]:] == 7.0).all()
        if w is not None:
            assert (w[b, :, (c.lens[b] if rows[b] else 0):] == 7.0).all()
    return O, lse, w


DECODE = [
    # lens, Lq, q_len, Hq, Hkv, d, page, S, T, mask
    ([1], 1, None, 1, 1, 64, 16, 64, 16, [0]),
    ([0, 1, 2], 1, [0, 1, 1], 4, 2, 128, 16, 64, 16, [1, 0]),
    ([517], 1, None, 32, 8, 128, 16, 128, 32, [0, 0, 1, 0, 0, 2, 1, 0]),
    ([5, 700, 64, 65, 63, 129], 1, None, 8, 2, 128, 64, 100, 37, [1, 0]),
    ([333, 80], 1, None, 3, 3, 64, 7, 50, 50, [2, 1, 0]),                      # MHA, odd pages
    ([200, 90, 1], 1, None, 12, 4, 128, 1, 64, 0, [0, 1, 2, 1]),               # one row to a page
    ([300, 41, 7, 130], 5, [5, 0, 3, 5], 8, 2, 128, 16, 32, 8, [0, 1]),        # rows cross segments; ragged; one idle
    ([260, 3], 4, [4, 3], 20, 1, 64, 100, 64, 64, [1]),                        # 80 rows to the KV head
    ([150], 33, None, 8, 4, 128, 48, 40, 10, [0, 1, 2, 0]),
    ([2, 5], 5, None, 4, 2, 128, 16, 16, 4, [0, 1]),                           # more rows than slots: the first see nothing
    ([5000, 1200], 1, None, 16, 2, 128, 64, 1 << 30, 0, [1, 0]),               # plainly causal
    ([9000, 17], 2, None, 64, 8, 128, 256, 4096, 1024, [1] * 8),
    ([4097], 1, None, 8, 1, 64, 128, 2048, 512, [1]),
    ([400, 90], 70, [70, 33], 4, 1, 128, 64, 128, 32, [0]),                    # 280 rows to the KV head
    ([300, 41], 40, [40, 0], 8, 2, 64, 16, 100, 20, [1, 2]),
    ([1500, 700, 130], 16, [16, 9, 16], 32, 8, 128, 64, 256, 64, [0, 1, 0, 1, 2, 1, 0, 1]),
    ([(37 * b) % 211 for b in range(300)], 1, [1 if (37 * b) % 211 and b % 7 else 0 for b in range(300)], 4, 2, 64, 16, 50, 20, [0, 1]),
    ([(37 * b) % 211 + 9 for b in range(200)], 9, [b % 10 for b in range(200)], 8, 2, 64, 16, 50, 20, [2, 1]),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "n%s_q%d_h%d_%d_d%d_p%d" % (max(c[0]), c[1], c[3], c[4], c[5], c[6]))
def test_decode_matches_the_definition(case, fp8):
    lens, Lq, q_len, Hq, Hkv, d, page, S, T, mask = case
    c = ref.Cache(lens, Hkv, d, page, fp8=fp8, seed=len(lens) + lens[-1])
    run_decode(c, rand_q(len(lens), Lq, Hq, d), S, T, mask, q_len=q_len)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "n%s_q%d_h%d_%d_d%d_p%d" % (max(c[0]), c[1], c[3], c[4], c[5], c[6]))
def test_decode_gathers_attention_weights(case, fp8):
    lens, Lq, q_len, Hq, Hkv, d, page, S, T, mask = case
    c = ref.Cache(lens, Hkv, d, page, fp8=fp8, seed=len(lens) + lens[-1])
    Q = rand_q(len(lens), Lq, Hq, d)
    O, lse, w = run_decode(c, Q, S, T, mask, q_len=q_len, want_weights=True)
    # added to what is there, in place, and the same from run to run
    acc = torch.rand(w.shape, generator=torch.Generator().manual_seed(3)).cuda()
    _, _, w3 = run_decode(c, Q, S, T, mask, q_len=q_len, weights=acc, want_weights=True)
    kept = acc.clone()
    sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, weights=acc, weights_out=acc,
                       q_len=None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda"), **c.dev, **c.scales)
    for b, n in enumerate(lens):
        m = n if (q_len is None or q_len[b]) else 0
        assert torch.equal(acc[b, :, :m], w3[b, :, :m]) and torch.equal(acc[b, :, m:], kept[b, :, m:])


@pytest.mark.parametrize("Lq,Hq,d,fp8", [(6, 4, 128, False), (6, 2, 64, False), (6, 12, 128, False), (40, 4, 128, False), (70, 4, 64, False),
                                         (6, 4, 128, True), (6, 12, 64, True), (20, 4, 128, True)])
def test_rows_nobody_sees_do_not_matter(Lq, Hq, d, fp8):
    # new row t must not feel the keys and values of the rows after it, whatever they hold; a local head not those before it
    lens, Hkv, page, S, T = [Lq + 64, Lq + 31], 2, 16, 32, 8
    mask = [0, 1]
    c = ref.Cache(lens, Hkv, d, page, fp8=fp8, seed=5)
    Q = rand_q(2, Lq, Hq, d)
    clean, lse, _ = run_decode(c, Q, S, T, mask)
    last = Lq - 2    # rows from this one on are spoiled
    bits = lambda x: x.view(torch.uint8) if fp8 else x
    for fill in ((0x7f, 0xff) if fp8 else (math.inf, -math.inf, math.nan, 3.0e38)):
        K, V = c.K.clone(), c.V.clone()
        for b, n in enumerate(lens):
            for j in range(n - Lq + last, n):
                bits(K)[c.table[b, j // page].long(), j % page] = fill
                bits(V)[c.table[b, j // page].long(), j % page] = fill
            low = min(ref.lowest_visible(n - Lq + t, S, T, 0, 0) for t in range(Lq))
            for j in range(0, low):
                bits(K)[c.table[b, j // page].long(), j % page, 0] = fill
                bits(V)[c.table[b, j // page].long(), j % page, 0] = fill
        w = torch.zeros(2, Hkv, c.max_pages * page, device="cuda")
        O, l2 = sa.seg_attn_decode(Q, K, V, S=S, T=T, head_past_mask=mask, weights_out=w, **c.dev, **c.scales)
        sa.poll_status()
        assert torch.equal(O[:, :last], clean[:, :last]) and torch.equal(l2[:, :, :last], lse[:, :, :last])
        assert not torch.isfinite(O[:, last:].float()).all()      # and those that see them do
        # only V is spoiled: the weights are what they were, and the rows that see them have what the sum has
        O, l2 = sa.seg_attn_decode(Q, c.K, V, S=S, T=T, head_past_mask=mask, **c.dev, **c.scales)
        assert torch.equal(l2, lse) and torch.equal(O[:, :last], clean[:, :last])
        if fp8 or not abs(fill) < math.inf:
            assert not torch.isfinite(O[:, last:].float()).any()


@pytest.mark.parametrize("Hq,d", [(2, 64), (20, 128), (40, 64), (44, 128)])
def test_rows_across_a_segment_border_do_not_feel_what_the_border_hides(Hq, d):
    # the first row of a segment sees the tail in front of it, the row before sees further back: infinities there reach one
    # of them only
    S, T, page = 32, 4, 16
    c = ref.Cache([66], 1, d, page, seed=8)      # rows 63 (old segment), 64 and 65 (new one)
    Q = rand_q(1, 3, Hq, d)
    clean, lse, _ = run_decode(c, Q, S, T, [0])
    K, V = c.K.clone(), c.V.clone()
    for j in (40, 59):                            # visible from 63, not from 64 on (which see 60..)
        K[c.table[0, j // page].long(), j % page] = math.nan
        V[c.table[0, j // page].long(), j % page] = math.inf
    O, l2 = sa.seg_attn_decode(Q, K, V, S=S, T=T, head_past_mask=[0], **c.dev)
    sa.poll_status()
    assert torch.equal(O[:, 1:], clean[:, 1:]) and torch.equal(l2[:, :, 1:], lse[:, :, 1:])
    assert not torch.isfinite(O[:, 0].float()).any()


@pytest.mark.parametrize("fp8,Lq", [(False, 2), (False, 8), (False, 16), (False, 32), (False, 48), (True, 2), (True, 16)])
def test_a_row_whose_scores_are_all_minus_infinity_weighs_nothing(Lq, fp8):
    # one query head's scores pass fp32's range downwards at every slot: O = 0, LSE = -inf, and the weights are the other rows'
    n, Hq, d, page, dead = 420, 4, 128, 16, 1
    c = ref.Cache([n], 1, d, page, fp8=fp8, seed=4)
    K = c.K.float()
    K[..., 0] = 100.0 if fp8 else 1.0e4
    K = K.to(c.K.dtype)
    Q = rand_q(1, Lq, Hq, d)
    Q[..., 0] = 0
    Q[0, Lq // 2, dead, 0] = -2.0e38
    if fp8:
        c.scales["k_scale"].fill_(16.0)      # times 100 times 2e38, over the root of 128
    w = torch.zeros(1, 1, c.max_pages * page, device="cuda")
    O, lse = sa.seg_attn_decode(Q, K, c.V, S=1 << 30, T=0, head_past_mask=[1], weights_out=w, **c.dev, **c.scales)
    sa.poll_status()
    assert not O[0, Lq // 2, dead].any() and lse[0, dead, Lq // 2] == -math.inf
    assert torch.isfinite(w).all()
    kw = {} if not fp8 else dict(k_scale=np.array([16.0]), v_scale=c.v_scale.double().numpy())
    Q[0, Lq // 2, dead] = 0                  # a row of equal weights instead, taken off the reference's sum
    want = ref.decode(f64(Q), K, c.V, c.table.numpy(), [n], [Lq], 1 << 30, 0, [1], d ** -0.5, page, **kw)
    e = n - Lq + Lq // 2
    want_w = want[4][0, 0]
    want_w[:e + 1] -= 1.0 / (e + 1)
    es = (d + 8) * ref.FP32 * want[3].max() + 2.0 ** -18
    assert abs(w.double().sum().item() - (Lq * Hq - 1)) <= 2 * es * Lq * Hq
    assert (np.abs(w[0, 0].cpu().double().numpy() - want_w) <= 2 * es * want_w + 4 * ref.FP32 * Lq * Hq).all()


def test_large_and_equal_scores():
    # scores of +-1e4 (one key wins outright) and keys that are all alike (every weight 1/n)
    c = ref.Cache([300], 2, 128, 16, seed=2)
    Q = rand_q(1, 1, 4, 128) * 300
    run_decode(c, Q, 1 << 30, 0, [1, 1])
    c.K[:] = 0.5
    run_decode(c, Q, 1 << 30, 0, [1, 1], want_weights=True)


@pytest.mark.parametrize("d,Lq,tail", [(64, 1, 0.01), (64, 4, 0.001), (64, 8, 0.01), (64, 16, 0.001), (128, 1, 0.001), (128, 8, 0.001), (128, 16, 0.01),
                                       (128, 24, 0.001)])
def test_small_weights_beside_a_dominant_key_keep_their_precision(d, Lq, tail):
    # 32K slots of an 8-bit cache whose first key takes all but `tail` of the weight and has no value of its own: what comes out
    # is the small weights' work.  Many sequences over the same pages, so that one block goes through (nearly) a whole sequence.
    n, B, Hkv, g, page = 32768, 448, 4, 4, 256
    gen = torch.Generator().manual_seed(d + Lq)
    k, v = 4 * torch.randn(n // page, page, Hkv, d, generator=gen), 4 * torch.randn(n // page, page, Hkv, d, generator=gen) + 4
    ks, vs = torch.full((Hkv,), 0.25), torch.full((Hkv,), 0.25)
    Q = torch.randn(B, Lq, Hkv * g, d, generator=gen)
    # element 0 is the first key's own: its score is what the others' sum needs to come to `tail`
    k[..., 0], k[0, 0], v[0, 0] = 0, 0, 0
    Q[..., 0], k[0, 0, :, 0] = 4.0, (math.log(n / tail) + 0.5) * d ** 0.5
    K, V = k.to(torch.float8_e4m3fn).cuda(), v.to(torch.float8_e4m3fn).cuda()
    Q = Q.bfloat16()
    table = torch.arange(n // page, dtype=torch.int32).expand(B, -1).contiguous()
    O, lse = sa.seg_attn_decode(Q.cuda(), K, V, table.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"), 1 << 30, 0, [1] * Hkv,
                                k_scale=ks.cuda(), v_scale=vs.cuda())
    sa.poll_status()
    some = [0, 1, 223, 447] if Lq == 1 else [5, 300]
    Or, lr, spread, terms, w = ref.decode(f64(Q[some]), K, V, table[some].numpy(), [n] * len(some), [Lq] * len(some), 1 << 30, 0, [1] * Hkv, d ** -0.5, page,
                                          k_scale=ks.double().numpy(), v_scale=vs.double().numpy())
    assert (w[:, :, 0] / (Lq * g) > 1 - 4 * tail).all() and (w[:, :, 0] / (Lq * g) < 1 - tail / 4).all()
    # as in check_decode, and half a step of an fp16 number below its normal range, 2^-25, where the largest weight is 2^13 at least
    es = (d + 8) * ref.FP32 * terms + 2.0 ** -18
    size = (np.abs(ref.rows_of(V, table[0].numpy(), n, page)) * 0.25).sum(0).repeat(g, 0)      # [Hq, d]
    bound = (ref.FP16 + 2 * es.transpose(0, 2, 1)[..., None]) * spread + 1.02 * ref.BF16 * np.abs(Or) + 2.0 ** -38 * size
    err = np.abs(f64(O[some]) - Or)
    assert (err <= bound).all(), float((err / bound).max())
    assert (np.abs(lse[some].cpu().double().numpy() - lr) <= es + 4 * ref.FP32 * np.abs(lr)).all()


@pytest.mark.parametrize("Hq", [4, 16, 64])
def test_scores_too_large_for_a_fraction(Hq):
    # scores of 2e9, whose fp32 steps are 128: a base is rounded by more than the slack, and nothing may overflow for it
    n, d, page = 300, 64, 16
    c = ref.Cache([n], 1, d, page, fp8=True, seed=2)
    K = c.K.clone()
    K.view(torch.uint8)[:] = torch.full((1,), 1.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
    for j, x in ((7, 448.0), (130, 448.0), (131, 416.0)):
        K[c.table[0, j // page].long(), j % page] = torch.full((1, d), x, device="cuda").to(torch.float8_e4m3fn)
    Q = torch.full((1, 1, Hq, d), 65536.0, dtype=torch.bfloat16, device="cuda")
    s = torch.full((1,), 8.0, device="cuda")
    O, lse = sa.seg_attn_decode(Q, K, c.V, c.dev["block_table"], c.dev["kv_len"], 1 << 30, 0, [1], k_scale=s, v_scale=s)
    sa.poll_status()
    # which of the two equal keys wins is within the scores' rounding; the row is their mean with some weights
    vals = ref.rows_of(c.V, c.table[0].numpy(), n, page)[[7, 130], 0] * 8.0
    slack = (2 * ref.FP16 + 1.02 * ref.BF16) * np.abs(vals).max(0)
    got = f64(O)[0, 0]
    assert (got >= vals.min(0) - slack).all() and (got <= vals.max(0) + slack).all()
    top = d * 65536.0 * 448 * 8 * d ** -0.5
    assert (np.abs(lse.cpu().double().numpy() - top) <= 8 * ref.FP32 * top).all()


@pytest.mark.parametrize("Lq,Hq,d,fp8", [(1, 8, 128, False), (4, 8, 64, False), (8, 8, 128, False), (16, 8, 128, False), (40, 8, 64, False),
                                         (1, 8, 64, True), (16, 8, 128, True), (40, 8, 64, True)])
def test_outputs_in_the_queries_place(Lq, Hq, d, fp8):
    # out may be Q; not where the gathered weights of many rows read Q again; never where a view shares some of its elements
    c = ref.Cache([900, 300], 2, d, 16, fp8=fp8, seed=9)
    Q = rand_q(2, Lq, Hq, d, pad_heads=1)
    many = Lq * Hq // 2 > 32 and not fp8
    call = lambda q, **kw: sa.seg_attn_decode(q, c.K, c.V, S=64, T=16, head_past_mask=[0, 1], **c.dev, **c.scales, **kw)
    for with_w in (False, True):
        w = [torch.zeros(2, 2, c.max_pages * 16, device="cuda") if with_w else None for _ in range(2)]
        O, lse = call(Q, weights_out=w[0])
        q = torch.cat([Q, Q.new_full((2, Lq, 1, d), 7.0)], 2)
        kept = q.clone()
        if many and with_w:
            with pytest.raises(sa.SegAttnError) as e:
                call(q[:, :, :Hq], out=q[:, :, :Hq], weights_out=w[1])
            assert e.value.status == 1 and torch.equal(q, kept) and not w[1].any()
            continue
        O2, l2 = call(q[:, :, :Hq], out=q[:, :, :Hq], weights_out=w[1])
        assert torch.equal(O, O2) and torch.equal(lse, l2) and (q[:, :, Hq] == 7.0).all()
        assert w[0] is None or torch.equal(w[0], w[1])
    q = torch.cat([Q, Q], 2)
    for out in (q[:, :, 1:Hq + 1], q[:, :, Hq - 1:2 * Hq - 1]):
        with pytest.raises(sa.SegAttnError):
            call(q[:, :, :Hq], out=out)
    O, lse = call(Q)
    O2, l2 = call(q[:, :, :Hq], out=q[:, :, Hq:])       # the other half of the same buffer
    assert O2.data_ptr() == q[:, :, Hq:].data_ptr() and torch.equal(O, O2) and torch.equal(lse, l2) and torch.equal(q[:, :, :Hq], Q)
    sa.poll_status()


def test_layouts_and_strides():
    lens = [130, 47]
    c = ref.Cache(lens, 4, 128, 16, seed=4, head_major=True)
    Q = rand_q(2, 3, 8, 128, pad_heads=2)          # a slice of a fused projection
    run_decode(c, Q, 64, 16, [0, 1, 2, 0], want_weights=True)
    # a block table that is a slice of a wider one
    wide = torch.full((2, c.max_pages + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.max_pages] = c.dev["block_table"]
    O1, l1 = sa.seg_attn_decode(Q, c.K, c.V, wide[:, :c.max_pages], c.dev["kv_len"], 64, 16, [0, 1, 2, 0])
    O2, l2 = sa.seg_attn_decode(Q, c.K, c.V, c.dev["block_table"], c.dev["kv_len"], 64, 16, [0, 1, 2, 0])
    assert torch.equal(O1, O2) and torch.equal(l1, l2)
    # an output of its own strides
    out = torch.zeros(2, 8, 3, 128, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    sa.seg_attn_decode(Q, c.K, c.V, c.dev["block_table"], c.dev["kv_len"], 64, 16, [0, 1, 2, 0], out=out)
    assert torch.equal(out, O2)


def test_the_shift_moves_positions_but_not_slots():
    lens, shift = [90, 40], [100, 0]
    c = ref.Cache(lens, 3, 64, 16, seed=6)
    run_decode(c, rand_q(2, 2, 6, 64), 64, 16, [0, 1, 2], shift=shift, want_weights=True)


def test_bad_numbers_are_reported_and_not_followed():
    c = ref.Cache([70, 40], 2, 128, 16, seed=7)
    Q = rand_q(2, 1, 4, 128)
    def second_is_right(O, lse):
        want = ref.decode(f64(Q), c.K, c.V, c.table.numpy(), c.lens, [0, 1], 64, 16, [1, 1], 128 ** -0.5, 16)
        ref.check_decode(O, lse, want, [0, 1], 128)

    for bad in (-1, c.K.shape[0], 1 << 30):
        t = c.table.clone()
        t[0, 2] = bad
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, t.cuda(), c.dev["kv_len"], 64, 16, [1, 1])
        with pytest.raises(sa.SegAttnError) as e:
            sa.poll_status()
        assert e.value.status == 1
        second_is_right(O, lse)
        want = ref.decode(f64(Q), c.K, c.V, t.numpy(), [70, 40], [1, 1], 64, 16, [1, 1], 128 ** -0.5, 16, bad_pages=(bad,)) \
            if bad < 0 else None
        if want is not None:
            ref.check_decode(O, lse, want, [1, 1], 128)
    for lens in ([c.max_pages * 16 + 1, 40], [-3, 40]):
        t = c.table.clone().clamp(min=0)
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, t.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), 64, 16, [1, 1])
        with pytest.raises(sa.SegAttnError):
            sa.poll_status()
        second_is_right(O, lse)
    for q in ([2, 1], [-1, 1]):
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, S=64, T=16, head_past_mask=[1, 1],
                                    q_len=torch.tensor(q, dtype=torch.int32, device="cuda"), **c.dev)
        with pytest.raises(sa.SegAttnError):
            sa.poll_status()
        second_is_right(O, lse)
    sa.poll_status()


def test_a_cache_without_pages_and_a_shared_page():
    for Lq, fp8 in ((1, False), (2, True), (40, False)):
        kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
        K = torch.empty(0, 16, 2, 64, device="cuda").to(kind)
        s = torch.ones(2, device="cuda") if fp8 else None
        w = torch.full((3, 2, 4), 7.0, device="cuda")
        O, lse = sa.seg_attn_decode(rand_q(3, Lq, 4, 64), K, K, torch.empty(3, 0, dtype=torch.int32, device="cuda"),
                                    torch.zeros(3, dtype=torch.int32, device="cuda"), 64, 16, [0, 1], weights_out=w, k_scale=s, v_scale=s)
        sa.poll_status()
        assert not O.any() and (lse == -math.inf).all() and (w == 7.0).all()
    c = ref.Cache([40, 50], 2, 64, 16, seed=2)      # both read the first sequence's first two pages
    c.table[1, :2] = c.table[0, :2]
    c.dev["block_table"] = c.table.cuda()
    run_decode(c, rand_q(2, 1, 4, 64), 1 << 30, 0, [1, 1])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Lq,Hq,max_pages", [(1, 4, 0), (9, 4, 0), (40, 4, 0), (1, 4, 1), (9, 4, 2), (40, 4, 3)])
def test_nothing_is_written_behind_the_workspace(Lq, Hq, max_pages, fp8):
    # the workspace is exactly as long as asked for; a cache without slots has no scores to keep
    B, Hkv, d, page = 3, 2, 64, 16
    c = ref.Cache([0] * B if max_pages == 0 else [max_pages * page] * B, Hkv, d, page, fp8=fp8, seed=1)
    table = c.dev["block_table"][:, :max_pages].contiguous()
    view = sa.paged._cache(c.K, c.V, table, c.dev["kv_len"], None, None, c.scales.get("k_scale"), c.scales.get("v_scale"))[0]
    need = sa.lib().seg_attn_decode_workspace_bytes(view, Lq, Hq, 1)
    buf = torch.full((need + (1 << 16),), 0x5a, dtype=torch.uint8, device="cuda")
    w = torch.full((B, Hkv, max_pages * page + 4), 7.0, device="cuda")
    sa.seg_attn_decode(rand_q(B, Lq, Hq, d), c.K, c.V, table, c.dev["kv_len"], 64, 16, [0, 1], weights_out=w, workspace=buf[:need], **c.scales)
    sa.poll_status()
    assert (buf[need:] == 0x5a).all() and (w[:, :, max_pages * page:] == 7.0).all()


def test_a_captured_step_follows_the_lengths():
    # one decoding step captured, replayed while the lengths, the table and the inputs change; two graphs side by side
    c = ref.Cache([200, 120], 2, 128, 16, seed=9)
    mask, S, T = [0, 1], 64, 16
    Q = rand_q(2, 1, 8, 128)
    w = torch.zeros(2, 2, c.max_pages * 16, device="cuda")
    sa.seg_attn_decode(Q, c.K, c.V, S=S, T=T, head_past_mask=mask, weights=w, weights_out=w, **c.dev)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        gr, q, acc = torch.cuda.CUDAGraph(), Q.clone(), torch.zeros_like(w)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(gr, stream=s):
            O, lse = sa.seg_attn_decode(q, c.K, c.V, S=S, T=T, head_past_mask=mask, weights_out=acc, **c.dev)
        graphs.append((gr, q, acc, O, lse, s))
    for n in ([200, 120], [1, 119], [65, 0], [150, 33]):
        c.dev["kv_len"].copy_(torch.tensor(n, dtype=torch.int32))
        for k, (gr, q, *_rest) in enumerate(graphs):
            q.copy_(rand_q(2, 1, 8, 128, seed=n[0] + k))
        torch.cuda.synchronize()
        for gr, *_rest, s in graphs:      # both at once
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for gr, q, acc, O, lse, s in graphs:
            a2 = torch.zeros_like(acc)
            O2, l2 = sa.seg_attn_decode(q, c.K, c.V, S=S, T=T, head_past_mask=mask, weights_out=a2, **c.dev)
            assert torch.equal(O, O2) and torch.equal(lse, l2)
            for b in range(2):
                assert torch.equal(acc[b, :, :n[b]], a2[b, :, :n[b]])
    sa.poll_status()


def test_a_call_on_a_given_stream_allocates_there():
    # results and workspaces of a call on another stream than the current one must not be handed out on the current one while
    # its kernels run: many calls on a side stream, their memory freed at once, while the current stream keeps allocating
    c = ref.Cache([3000, 2000], 2, 128, 64, seed=12)
    Q = rand_q(2, 1, 16, 128)
    w = torch.rand(2, 2, c.max_pages * 64, device="cuda")
    want = sa.seg_attn_decode(Q, c.K, c.V, S=64, T=16, head_past_mask=[1, 1], **c.dev)
    table = sa.rope_table_scaled(8, 128)
    turned = sa.rope_rotate(Q, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(30):
        got.append(sa.seg_attn_decode(Q, c.K, c.V, S=64, T=16, head_past_mask=[1, 1], stream=side, **c.dev) + (sa.rope_rotate(Q, table, stream=side),))
        torch.full((1 << 22,), math.nan, device="cuda")
    side.synchronize()
    torch.cuda.synchronize()
    for O, lse, y in got:
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1]) and torch.equal(y, turned)
    sa.poll_status()


def test_offsets_past_32_bits():
    # pages 2^31 + elements apart
    page, Hkv, d = 16, 2, 128
    gap = (1 << 31) + 4096
    buf = torch.zeros(gap + page * Hkv * d, dtype=torch.bfloat16, device="cuda")
    K = buf.as_strided((2, page, Hkv, d), (gap, Hkv * d, d, 1))
    small = torch.randn(2, page, Hkv, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    K.copy_(small)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    n = torch.tensor([29], dtype=torch.int32, device="cuda")
    Q = rand_q(1, 1, 4, d)
    a = sa.seg_attn_decode(Q, K, K, table, n, 1 << 30, 0, [1, 1])
    b = sa.seg_attn_decode(Q, small, small, table, n, 1 << 30, 0, [1, 1])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    new = torch.randn(1, 1, Hkv, d, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    n2 = torch.tensor([7], dtype=torch.int32, device="cuda")
    sa.kv_append(new, new, K, small, table, n2)
    assert torch.equal(K[1, 6], new[0, 0]) and torch.equal(small[1, 6], new[0, 0])
    del K, buf


# ---- append ----------------------------------------------------------------------------------------------------------

APPEND = [
    # lens (after), Lq, q_len, Hq, Hkv, d, page, rot, layout
    ([1], 1, None, 2, 1, 64, 16, 64, "half"),
    ([5, 33, 20], 5, [5, 0, 3], 8, 2, 128, 7, 128, "interleaved"),
    ([300, 260], 256, None, 6, 3, 128, 64, 32, "half"),
    ([100, 17], 17, [9, 17], 4, 4, 64, 16, 48, "interleaved"),
    ([40], 40, None, 0, 2, 128, 1, 96, "half"),          # keys alone
    ([40, 39], 8, None, 0, 2, 64, 48, 0, "half"),        # no rotation
    ([700, 500, 2], 500, [500, 500, 2], 32, 8, 128, 100, 64, "interleaved"),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: "n%d_q%d_d%d_p%d_r%d" % (max(c[0]), c[1], c[5], c[6], c[7]))
def test_append_matches_the_definition(case, fp8):
    lens, Lq, q_len, Hq, Hkv, d, page, rot, layout = case
    B = len(lens)
    c = ref.Cache(lens, Hkv, d, page, fp8=fp8, seed=lens[0])
    g = torch.Generator().manual_seed(77)
    mk = lambda H: (torch.randn(B, Lq, H + 1, d, generator=g) * 30).bfloat16().cuda()[:, :, :H]
    Kn, Vn = mk(Hkv), mk(Hkv)
    if fp8:
        Vn[0, 0, 0, :2] = torch.tensor([math.inf, math.nan])     # saturates, stays NaN
    Q = mk(Hq) if Hq else None
    rows = [Lq] * B if q_len is None else q_len
    shift = [3 * b for b in range(B)]
    table = sa.rope_table_scaled(max(lens) + 3 * B, rot, amplitude=1.25) if rot else None
    qo = torch.full_like(Q, 7.0) if Hq else None
    K0, V0 = c.K.clone(), c.V.clone()
    sa.kv_append(Kn, Vn, c.K, c.V, table=table, layout=layout, Q=Q, q_out=qo, pos_shift=torch.tensor(shift, dtype=torch.int32, device="cuda"),
                 q_len=None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda"), **c.dev, **c.scales)
    sa.poll_status()
    bits = lambda t: t.view(torch.uint8) if fp8 else t.view(torch.int16)
    want_k, want_v = bits(K0).clone(), bits(V0).clone()
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    for b in range(B):
        for t in range(rows[b]):
            slot = lens[b] - rows[b] + t
            tab = table[slot + shift[b]].cpu().numpy() if rot else None
            k, v = Kn[b, t].float().cpu().numpy(), Vn[b, t].float().cpu().numpy()
            if rot:      # every product and sum rounded to 32 bits, as the kernel documents: the same bits
                k = ref.rotate(k, tab, layout)
            k, v = torch.from_numpy(k), torch.from_numpy(v)
            if fp8:
                k, v = (k * (1 / c.k_scale)[:, None]).clamp(-448, 448), (v * (1 / c.v_scale)[:, None]).clamp(-448, 448)
            at = c.table[b, slot // page].long(), slot % page
            want_k[at], want_v[at] = bits(k.to(kind)).cuda(), bits(v.to(kind)).cuda()
            if Hq:
                q64 = ref.rotate(Q[b, t].float().cpu().double().numpy(), tab.astype(np.float64), layout)
                size = 1.25 * np.abs(Q[b, t].float().cpu().double().numpy()).max()
                assert (np.abs(f64(qo[b, t]) - q64) <= ref.BF16 * np.abs(q64) + 8 * ref.FP32 * size).all()
                assert torch.equal(qo[b, t].cpu(), torch.from_numpy(ref.rotate(Q[b, t].float().cpu().numpy(), tab, layout)).bfloat16())
        if Hq:
            assert (qo[b, rows[b]:] == 7.0).all()
    if fp8:      # any NaN is as good as another
        nan = lambda x: torch.where((x & 0x7f) == 0x7f, 0x7f, x)
        assert torch.equal(nan(bits(c.K)), nan(want_k)) and torch.equal(nan(bits(c.V)), nan(want_v))
    else:
        assert torch.equal(bits(c.K), want_k) and torch.equal(bits(c.V), want_v)


@pytest.mark.parametrize("scale", [1.0, 0.0371, 3.0, 1.0e-3, 2.0 ** -127, 1.0e-38, 2.0e38])
def test_eight_bit_values_are_rounded_to_nearest_even(scale):
    # values on and around the borders between two e4m3 values, times the scale's inverse in fp32
    grid = torch.arange(0, 0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    border = (grid[1:] + grid[:-1]) / 2 * scale
    near = torch.cat([border, grid * scale, border * (1 + 2.0 ** -9), border * (1 - 2.0 ** -9), torch.tensor([500.0 * scale, 1e30, 3e38, 0.0])])
    x = near.to(torch.bfloat16)
    x = torch.cat([x, -x])
    x = torch.cat([x, x.new_zeros(-len(x) % 128)]).reshape(1, -1, 1, 128).cuda()
    n = x.shape[1]
    pages = torch.zeros(2, 16, 1, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    assert n <= 16
    s = torch.tensor([scale], device="cuda")
    sa.kv_append(x, x, pages[:1], pages[1:], torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"),
                 k_scale=s, v_scale=s)
    sa.poll_status()
    want = (x[0].cpu().float() * (1 / torch.tensor(scale))).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(pages[0, :n].view(torch.uint8).cpu(), want) and torch.equal(pages[1, :n].view(torch.uint8).cpu(), want)


def test_append_in_place_and_bad_numbers():
    c = ref.Cache([20, 30], 2, 128, 16, seed=1)
    mk = lambda H: torch.randn(2, 4, H, 128, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    Kn, Vn, Q = mk(2), mk(2), mk(4)
    table = sa.rope_table(40, 128)
    want = sa.kv_append(Kn, Vn, c.K, c.V, table=table, Q=Q, **c.dev)
    Q2 = Q.clone()
    assert sa.kv_append(Kn, Vn, c.K, c.V, table=table, Q=Q2, q_out=Q2, **c.dev) is Q2 and torch.equal(Q2, want)
    sa.poll_status()
    K0, V0 = c.K.clone(), c.V.clone()
    bits = lambda t: t.view(torch.int16)

    def refused(**kw):
        K, V = K0.clone(), V0.clone()
        args = dict(c.dev, **kw)
        sa.kv_append(Kn * 2, Vn * 2, K, V, table=args.pop("table", table), Q=Q, **args)
        with pytest.raises(sa.SegAttnError) as e:
            sa.poll_status()
        assert e.value.status == 1
        return K, V

    at = lambda x, b, j: x[c.table[b, j // 16].long(), j % 16]
    t = c.table.clone()
    t[1, 1] = 99          # rows 26..29 of sequence 1 lie in its second page
    K, V = refused(block_table=t.cuda())
    assert torch.equal(bits(at(K, 1, 27)), bits(at(K0, 1, 27))) and torch.equal(at(V, 0, 17), Vn[0, 1] * 2)
    K, V = refused(table=table[:28])                      # positions 28 and 29 are not in the table
    assert torch.equal(bits(at(V, 1, 28)), bits(at(V0, 1, 28))) and torch.equal(at(V, 1, 27), Vn[1, 1] * 2)
    K, V = refused(kv_len=torch.tensor([20, 2], dtype=torch.int32, device="cuda"))     # four new rows, two slots
    assert torch.equal(at(V, 1, 0), Vn[1, 2] * 2) and torch.equal(at(V, 1, 1), Vn[1, 3] * 2)
    sa.poll_status()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rotated", [False, True])
def test_append_writes_no_row_in_another_s_place(rotated, fp8):
    # lengths past the table's capacity, below zero, more new rows than were given, a negative shift: rows without a place are
    # left out, the others go to their own slots, and every row that was there keeps its bits
    Hkv, d, page, Lq, pages = 2, 64, 8, 4, 5
    cap = page * pages
    g = torch.Generator().manual_seed(8)
    new = [torch.randn(2, Lq, Hkv, d, generator=g).bfloat16().cuda() for _ in range(2)]
    table = sa.rope_table_scaled(3 * cap, 32) if rotated else None
    low, high = -(1 << 31), (1 << 31) - 1
    for n, q_len, shift in ((cap + 1, None, None), (cap + 3, None, None), (cap + 4, None, None), (cap + 5, 2, None), (high, None, 5), (low, None, None),
                            (-1, None, None), (3, None, None), (cap, 5, None), (cap - 7, high, None), (20, -1, None), (20, low, None), (cap + 1, 0, None),
                            (20, None, -3), (20, None, low), (20, 4, 2)):
        c = ref.Cache([cap, cap], Hkv, d, page, fp8=fp8, seed=3)
        bits = lambda t: t.view(torch.uint8) if fp8 else t.view(torch.int16)
        K0, V0 = bits(c.K).clone(), bits(c.V).clone()
        i32 = lambda x, other: None if x is None else torch.tensor([x, other], dtype=torch.int32, device="cuda")
        sa.kv_append(new[0], new[1], c.K, c.V, c.dev["block_table"], i32(n, cap), table=table, q_len=i32(q_len, Lq), pos_shift=i32(shift, 0), **c.scales)
        rows = Lq if q_len is None else q_len
        valid = 0 <= rows <= Lq and not (rotated and shift is not None and shift < 0)
        here = [t for t in range(Lq) if valid and t < rows and 0 <= n - rows + t < cap]
        bad = not valid or (shift is not None and shift < 0) or len(here) < rows
        if bad and not (shift is not None and shift < 0 and not rotated):
            with pytest.raises(sa.SegAttnError) as e:
                sa.poll_status()
            assert e.value.status == 1
        elif not bad:
            sa.poll_status()
        else:      # a shift that nothing uses may be reported or not
            try:
                sa.poll_status()
            except sa.SegAttnError:
                pass
        # what the rows that have a place should be: the same rows appended alone, all numbers in range
        want = ref.Cache([cap, cap], Hkv, d, page, fp8=fp8, seed=3)
        for b, ts in ((0, here), (1, list(range(Lq)))):
            for t in ts:
                slot = (n - rows + t) if b == 0 else cap - Lq + t
                one = dict(block_table=want.dev["block_table"][b:b + 1], kv_len=torch.tensor([slot + 1], dtype=torch.int32, device="cuda"))
                sh = torch.tensor([shift if b == 0 and shift is not None and shift >= 0 else 0], dtype=torch.int32, device="cuda")
                sa.kv_append(new[0][b:b + 1, t:t + 1], new[1][b:b + 1, t:t + 1], want.K, want.V, table=table, pos_shift=sh, **one, **want.scales)
        sa.poll_status()
        assert torch.equal(bits(c.K), bits(want.K)) and torch.equal(bits(c.V), bits(want.V)), (n, q_len, shift)
        touched = torch.zeros(c.K.shape[0], page, dtype=torch.bool, device="cuda")
        for b, ts in ((0, here), (1, list(range(Lq)))):
            for t in ts:
                slot = (n - rows + t) if b == 0 else cap - Lq + t
                touched[c.table[b, slot // page].long(), slot % page] = True
        assert torch.equal(bits(c.K)[~touched], K0[~touched]) and torch.equal(bits(c.V)[~touched], V0[~touched])
    sa.poll_status()


# ---- eviction ---------------------------------------------------------------------------------------------------------

EVICT = [
    # lens, Hkv, d, page, sink, recent, heavy
    ([100], 2, 128, 16, 4, 20, 16),
    ([40, 41, 39, 0, 1], 3, 64, 7, 4, 20, 16),
    ([700, 2500], 2, 64, 64, 0, 0, 333),
    ([1025, 1024, 3000], 1, 128, 16, 1, 1000, 0),
    ([5000, 300], 8, 128, 100, 16, 100, 1500),
    ([64], 1, 64, 1, 0, 1, 0),
    ([20000, 9000], 2, 64, 256, 5, 777, 4001),
    ([70000], 2, 64, 256, 16, 2048, 3000),
]


def make_weights(kind, B, Hkv, W, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.rand(B, Hkv, W, generator=g)
    if kind == "ties":
        w = (w * 5).floor() / 5
    elif kind == "flat":
        w = torch.zeros_like(w)
    elif kind == "wide":
        w = torch.exp2((w - 0.5) * 200) * torch.where(torch.rand(w.shape, generator=g) < 0.1, -1.0, 1.0)
    elif kind == "odd":
        r = torch.rand(w.shape, generator=g)
        w[r < 0.1], w[(r >= 0.1) & (r < 0.2)] = math.nan, math.inf
        w[(r >= 0.2) & (r < 0.3)], w[(r >= 0.3) & (r < 0.4)] = -0.0, 0.0
        w[(r >= 0.4) & (r < 0.45)] = -math.inf
    return w


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "flat", "wide", "odd"])
@pytest.mark.parametrize("case", EVICT, ids=lambda c: "n%d_h%d_d%d_p%d_%d_%d_%d" % (max(c[0]), *c[1:]))
def test_evict_matches_the_definition(case, kind, fp8):
    lens, Hkv, d, page, sink, recent, heavy = case
    budget, B = sink + recent + heavy, len(lens)
    per = -(-budget // page)
    c = ref.Cache(lens, Hkv, d, page, fp8=fp8, seed=budget, spare=B * per + 2)
    dst = torch.tensor(c.spare[:B * per], dtype=torch.int32).reshape(B, per)
    W = c.max_pages * page
    if budget > W:
        pytest.skip("budget past the cache")
    w = make_weights(kind, B, Hkv, W, seed=7).cuda()
    shift = torch.arange(B, dtype=torch.int32, device="cuda") * 10
    bits = lambda t: t.view(torch.uint8) if fp8 else t.view(torch.int16)
    K0, V0 = bits(c.K).clone(), bits(c.V).clone()
    idx, n2, s2, w2 = sa.kv_evict(w, c.K, c.V, dst_table=dst.cuda(), sink=sink, recent=recent, heavy=heavy, pos_shift=shift, **c.dev)
    sa.poll_status()
    want_k, want_v, want_w = K0.clone(), V0.clone(), torch.zeros(B, Hkv, W)
    wc = w.cpu()
    for b, n in enumerate(lens):
        for h in range(Hkv):
            keep = ref.evict_choice(wc[b, h].tolist(), n, sink, recent, heavy)
            got = idx[b, h].cpu().tolist()
            assert got == keep + [-1] * (budget - len(keep))
            want_w[b, h, :len(keep)] = wc[b, h, keep]
            src, r = torch.tensor(keep, dtype=torch.long), torch.arange(len(keep))
            a, z = c.table[b, src // page].long(), dst[b, r // page].long()
            want_k[z.cuda(), (r % page).cuda(), h] = K0[a.cuda(), (src % page).cuda(), h]
            want_v[z.cuda(), (r % page).cuda(), h] = V0[a.cuda(), (src % page).cuda(), h]
        m = min(n, budget)
        assert (int(n2[b]), int(s2[b])) == (m, 10 * b + n - m)
    assert torch.equal(bits(c.K), want_k) and torch.equal(bits(c.V), want_v)
    assert torch.equal(w2.cpu().view(torch.int32), want_w.view(torch.int32))


def test_evict_in_place_lengths_and_bad_pages():
    c = ref.Cache([200, 50], 2, 128, 16, seed=3, spare=12)
    dst = torch.tensor(c.spare[:10], dtype=torch.int32).reshape(2, 5).cuda()
    w = torch.rand(2, 2, c.max_pages * 16, device="cuda")
    shift = torch.tensor([7, 0], dtype=torch.int32, device="cuda")
    n = c.dev["kv_len"].clone()
    a = sa.kv_evict(w, c.K, c.V, c.dev["block_table"], n, dst, 2, 30, 20, pos_shift=shift, kv_len_out=n, pos_shift_out=shift)
    sa.poll_status()
    assert n.tolist() == [52, 50] and shift.tolist() == [155, 0] and a[1] is n and a[2] is shift
    # a source page that is none: its rows come out zero; a destination that is none: its rows are not written
    t = c.table.clone()
    t[0, 0] = -5
    K, V = c.K.clone(), c.V.clone()
    b = sa.kv_evict(w, K, V, t.cuda(), c.dev["kv_len"], dst, 2, 30, 20)
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 1 and torch.equal(a[0], b[0])
    assert not K[dst[0, 0].long(), 0].any() and not V[dst[0, 0].long(), 1].any()
    assert torch.equal(K[dst[1, 0].long()], c.K[dst[1, 0].long()])
    d2 = dst.clone()
    d2[1, 1] = c.K.shape[0]
    K, V = c.K.clone().fill_(9), c.V.clone().fill_(9)
    sa.kv_evict(w, K, V, c.dev["block_table"], c.dev["kv_len"], d2, 2, 30, 20)
    with pytest.raises(sa.SegAttnError):
        sa.poll_status()
    with pytest.raises(sa.SegAttnError):        # no budget at all, more than the destination holds
        sa.kv_evict(w, K, V, c.dev["block_table"], c.dev["kv_len"], dst, 0, 0, 0)
    with pytest.raises(sa.SegAttnError):
        sa.kv_evict(w, K, V, c.dev["block_table"], c.dev["kv_len"], dst, 10, 50, 21)
    with pytest.raises(sa.SegAttnError):        # the weights may not be compacted in place
        sa.kv_evict(w, K, V, c.dev["block_table"], c.dev["kv_len"], dst, 2, 30, 20, weights_out=w)
    sa.poll_status()


# ---- together -----------------------------------------------------------------------------------------------------------

def test_prefill_then_decode_continues_the_sequence():
    # a prompt through the streamed prefill and into pages segment by segment, then token by token: every row is that of the
    # oracle's attention over the whole sequence (keys and queries rotated at their global positions)
    import oracle
    from util import assert_fwd_close
    B, Hq, Hkv, d, S, T, page, prompt, total = 2, 8, 4, 128, 64, 24, 16, 150, 200
    mask = [0, 1, 2, 1]
    g = torch.Generator().manual_seed(11)
    mk = lambda H: torch.randn(B, total, H, d, generator=g).bfloat16().cuda()
    Q, K, V = mk(Hq), mk(Hkv), mk(Hkv)
    table = sa.rope_table_scaled(total, 64, kind="by_parts", factor=4.0, trained_len=64.0, turns_lo=1.0, turns_hi=8.0)
    Qr, Kr = sa.rope_rotate(Q, table, layout="interleaved"), sa.rope_rotate(K, table, layout="interleaved")
    O_want, L_want = oracle.fwd(f64(Qr), f64(Kr), f64(V), S, T, mask)
    max_pages = -(-total // page)
    pages = torch.zeros(2 * B * max_pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    Kp, Vp = pages[:B * max_pages], pages[B * max_pages:]
    bt = torch.randperm(B * max_pages, generator=g).int().reshape(B, max_pages).cuda()
    n = torch.zeros(B, dtype=torch.int32, device="cuda")
    pf = sa.Prefill(B, S, T, Hq, Hkv, d, max_len=S * 4, head_past_mask=mask)
    wide = lambda x, p0, m: torch.cat([x[:, p0:p0 + m], x.new_zeros(B, S - m, *x.shape[2:])], 1)[:, :m]    # the strides of a full segment
    for p0 in range(0, prompt, S):
        m = min(S, prompt - p0)
        n += m
        q = sa.kv_append(K[:, p0:p0 + m], V[:, p0:p0 + m], Kp, Vp, bt, n, table=table, layout="interleaved", Q=Q[:, p0:p0 + m])
        assert torch.equal(q, Qr[:, p0:p0 + m])
        O, lse = pf.step(wide(q, 0, m), wide(Kr, p0, m), wide(V, p0, m))
        assert_fwd_close(O, lse, O_want[:, p0:p0 + m], L_want[:, :, p0:p0 + m], "prefill")
    pf.close()
    at = prompt
    for m in (1, 1, 1, 3, 1, 20, 1, 1, 21):
        n += m
        q = sa.kv_append(K[:, at:at + m], V[:, at:at + m], Kp, Vp, bt, n, table=table, layout="interleaved", Q=Q[:, at:at + m])
        O, lse = sa.seg_attn_decode(q, Kp, Vp, bt, n, S, T, mask)
        assert_fwd_close(O, lse, O_want[:, at:at + m], L_want[:, :, at:at + m], "decode")
        at += m
    assert at == total
    sa.poll_status()


def test_decode_evict_decode():
    # weights gathered over some steps, an eviction that keeps the last S + T rows, more steps: local and own-segment heads go
    # on as if nothing had happened, heads with past access attend over what was kept
    B, Hq, Hkv, d, S, T, page = 2, 6, 3, 64, 32, 8, 16
    mask = [0, 1, 2]
    sink, recent, heavy = 2, S + T, 20
    budget, steps, more = sink + recent + heavy, 6, 10
    lens = [150, 90]
    final = [x + steps + more for x in lens]
    c = ref.Cache(final, Hkv, d, page, seed=21, spare=12)      # the rows of all steps are in their slots already
    W = c.max_pages * page
    w = torch.zeros(B, Hkv, W, device="cuda")
    want_w = np.zeros((B, Hkv, W))
    for k in range(1, steps + 1):
        n = [x + k for x in lens]
        Q = rand_q(B, 1, Hq, d, seed=k)
        sa.seg_attn_decode(Q, c.K, c.V, c.dev["block_table"], torch.tensor(n, dtype=torch.int32, device="cuda"), S, T, mask, weights=w, weights_out=w)
        want_w += ref.decode(f64(Q), c.K, c.V, c.table.numpy(), n, [1] * B, S, T, mask, d ** -0.5, page)[4]
    sa.poll_status()
    assert np.abs(w.cpu().double().numpy() - want_w).max() < 1e-4
    n = torch.tensor([x + steps for x in lens], dtype=torch.int32, device="cuda")
    dst = torch.full((B, 6), -1, dtype=torch.int32)
    dst[0], dst[1] = torch.tensor(c.spare[:6]), torch.tensor(c.spare[6:12])
    dst = dst.cuda()
    idx, n2, shift, w2 = sa.kv_evict(w, c.K, c.V, c.dev["block_table"], n, dst, sink, recent, heavy)
    sa.poll_status()
    kept = [[ref.evict_choice(w[b, h].tolist(), lens[b] + steps, sink, recent, heavy) for h in range(Hkv)] for b in range(B)]
    assert [[idx[b, h].tolist() for h in range(Hkv)] for b in range(B)] == kept and n2.tolist() == [budget, budget]
    full = [(ref.rows_of(c.K, c.table[b].numpy(), final[b], page), ref.rows_of(c.V, c.table[b].numpy(), final[b], page)) for b in range(B)]
    for k in range(1, more + 1):
        rows = [torch.from_numpy(np.stack([full[b][x][lens[b] + steps + k - 1] for b in range(B)]))[:, None].bfloat16().cuda() for x in (0, 1)]
        n2 += 1
        sa.kv_append(rows[0], rows[1], c.K, c.V, dst, n2, pos_shift=shift)
        Q = rand_q(B, 1, Hq, d, seed=100 + k)
        O, lse = sa.seg_attn_decode(Q, c.K, c.V, dst, n2, S, T, mask, pos_shift=shift, weights=w2, weights_out=w2)
        for b in range(B):
            p = lens[b] + steps + k - 1
            for h in range(Hkv):
                low = ref.lowest_visible(p, S, T, mask[h], 0)
                see = list(range(low, p + 1)) if mask[h] != 1 else kept[b][h] + list(range(lens[b] + steps, p + 1))
                for q in range(2 * h, 2 * h + 2):
                    s = d ** -0.5 * full[b][0][see, h] @ f64(Q)[b, 0, q]
                    e = np.exp(s - s.max())
                    o = e / e.sum() @ full[b][1][see, h]
                    spread = e / e.sum() @ np.abs(full[b][1][see, h])
                    assert abs(float(lse[b, q, 0]) - (s.max() + math.log(e.sum()))) < 1e-4
                    assert (np.abs(f64(O)[b, 0, q] - o) <= (ref.BF16 + 1e-4) * spread + 1.02 * ref.BF16 * np.abs(o)).all()
    sa.poll_status()
    new = w2[:, :, budget:budget + more].sum((0, 2))
    assert (new > 0).all() and not w2[:, :, budget + more:].any()


def test_a_captured_decoding_loop_with_an_eviction():
    # one graph: a token appended, attended over, weights gathered, the length moved on; another: an eviction into the spare
    # pages.  Replayed against the same calls made one by one
    B, Hq, Hkv, d, page, S, T = 2, 8, 2, 128, 16, 32, 8
    mask, sink, recent, heavy = [0, 1], 1, S + T, 6
    table = sa.rope_table_scaled(400, 64, kind="linear", factor=2.0)
    g = torch.Generator().manual_seed(31)
    steps = [[torch.randn(B, 1, H, d, generator=g).bfloat16().cuda() for H in (Hkv, Hkv, Hq)] for _ in range(14)]

    def make():
        c = ref.Cache([60, 75], Hkv, d, page, seed=13, spare=12, max_pages=6)
        c.table[0, 4], c.table[1, 5] = c.spare[10], c.spare[11]      # room for the new rows
        x = dict(c=c, K=c.K, V=c.V, bt=c.table.clone().cuda(), n=c.dev["kv_len"].clone(), shift=torch.zeros(B, dtype=torch.int32, device="cuda"),
                 w=torch.zeros(B, Hkv, 110, device="cuda"), w2=torch.zeros(B, Hkv, 110, device="cuda"), k=steps[0][0].clone(), v=steps[0][1].clone(),
                 q=steps[0][2].clone(), dst=torch.tensor(c.spare[:10], dtype=torch.int32).reshape(B, 5).cuda())
        x["bt2"] = torch.full((B, 6), -1, dtype=torch.int32, device="cuda")
        x["bt2"][:, :5] = x["dst"]
        return x

    def token(x, bt, w, stream=None):
        x["n"] += 1
        q = sa.kv_append(x["k"], x["v"], x["K"], x["V"], bt, x["n"], table=table, Q=x["q"], pos_shift=x["shift"], stream=stream)
        return sa.seg_attn_decode(q, x["K"], x["V"], bt, x["n"], S, T, mask, pos_shift=x["shift"], weights=w, weights_out=w, stream=stream)

    def evict(x, stream=None):
        return sa.kv_evict(x["w"], x["K"], x["V"], x["bt"], x["n"], x["dst"], sink, recent, heavy, pos_shift=x["shift"], weights_out=x["w2"],
                           kv_len_out=x["n"], pos_shift_out=x["shift"], stream=stream)

    def feed(x, k):
        for name, t in zip(("k", "v", "q"), steps[k]):
            x[name].copy_(t)

    one, rep = make(), make()
    outs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                  # the direct calls on a stream of their own, given by name
        for k in range(14):
            feed(one, k)
            if k == 3:
                idx = evict(one, stream=side)[0]
            O, lse = token(one, one["bt"] if k < 3 else one["bt2"], one["w"] if k < 3 else one["w2"], stream=side)
            outs.append((O.clone(), lse.clone()))
    side.synchronize()
    start = {n: rep[n].clone() for n in ("n", "shift", "w", "w2")}
    K0, V0 = rep["K"].clone(), rep["V"].clone()
    graphs = []
    for f in (lambda: token(rep, rep["bt"], rep["w"]), lambda: evict(rep), lambda: token(rep, rep["bt2"], rep["w2"])):
        f()                                        # once outside, then the state put back
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr):
            res = f()
        graphs.append((gr, res))
    for n, t in start.items():
        rep[n].copy_(t)
    rep["K"].copy_(K0)
    rep["V"].copy_(V0)
    for k in range(14):
        feed(rep, k)
        if k == 3:
            graphs[1][0].replay()
            assert torch.equal(graphs[1][1][0], idx)
        gr, (O, lse) = graphs[0 if k < 3 else 2]
        gr.replay()
        assert torch.equal(O, outs[k][0]) and torch.equal(lse, outs[k][1]), k
    sa.poll_status()
    for n in ("n", "shift", "w2"):
        assert torch.equal(one[n], rep[n]), n
    assert one["n"].tolist() == [sink + recent + heavy + 11] * 2 and not one["w2"][:, :, 96:].any()
    for b in range(B):
        assert torch.equal(torch.isnan(one["K"].float()), torch.isnan(rep["K"].float()))
