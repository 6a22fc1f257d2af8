"""What a decoding loop relies on from one call to the next: means that follow rescaled rows, free lists of empty batches, scales that
are carried along or refused, numbers at the ends of their types."""
import math

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


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(300 + seed)).bfloat16().cuda()


def refused():
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 1


def fresh_means(c, block):
    n_pages, page, Hkv, d = c.K.shape
    return torch.full((n_pages, page // block, Hkv, d), 9, dtype=torch.int8, device="cuda"), torch.full((n_pages, page // block, Hkv), 7.0, device="cuda")


def same_means(c, block, got, lens):
    """The means of all full blocks are those of the rows that the cache holds now."""
    X = br.dequantised(c.K, c.scales["k_scale"])
    for b, n in enumerate(lens):
        for j in range(n // block):
            at, row = int(c.table[b, j * block // c.page]), j * block % c.page
            q, s = br.means(X[at, row:row + block], block)
            assert np.array_equal(got[0][at, row // block].cpu().numpy(), q) and np.array_equal(got[1][at, row // block].cpu().numpy(), s), (b, j)


@pytest.mark.parametrize("d,page,rows,block", [(64, 64, 64, 16), (128, 128, 128, 32), (128, 128, 64, 32), (64, 128, 32, 16), (64, 128, 64, 128), (128, 96, 32, 32)])
def test_means_follow_rows_that_an_append_rescales(d, page, rows, block):
    # keys grow along the sequence, so that tokens raise the scales of half-filled blocks again and again; steps of one token are captured
    # and replayed, those of several run as they come, and idle sequences stay as they are
    lens, Hkv = [0, 0, 0], 2
    c = br.ScaledCache([300] * 3, Hkv, d, page, rows, seed=1)
    means = fresh_means(c, block)
    n = ints(lens)
    kw = dict(block_table=c.dev["block_table"], kv_len=n)

    def step(K, V, q):
        sa.kv_append(K, V, c.K, c.V, q_len=q, **kw, **c.scales)
        sa.blocks_summarise(c.K, c.dev["block_table"], n, K.shape[1], *means, q_len=q, k_scale=c.scales["k_scale"])

    graphs = {}
    for Lq in (1, 9):
        K, V, q = rand(3, Lq, Hkv, d), rand(3, Lq, Hkv, d), ints([0] * 3)
        step(K, V, q)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(K, V, q)
        graphs[Lq] = gr, K, V, q
    for k in range(40):
        Lq = 1 if k % 4 else 9
        gr, K, V, q = graphs[Lq]
        new = [min(Lq, 300 - x) if (k + b) % 5 else 0 for b, x in enumerate(lens)]
        lens = [x + y for x, y in zip(lens, new)]
        for t, s in ((K, 2 * k), (V, 2 * k + 1)):
            t.copy_(rand(*t.shape, seed=s) * 2.0 ** (k // 3))
        n.copy_(ints(lens))
        q.copy_(ints(new))
        gr.replay()
    same_means(c, block, means, lens)
    for k, Lq in enumerate((70, 33, 5)):
        new = [min(Lq, 300 - x) for x in lens]
        lens = [x + y for x, y in zip(lens, new)]
        n.copy_(ints(lens))
        step(rand(3, Lq, Hkv, d, seed=90 + k) * 2.0 ** (14 + 2 * k), rand(3, Lq, Hkv, d, seed=95 + k), ints(new))
        same_means(c, block, means, lens)
    sa.poll_status()


def test_an_empty_batch_keeps_its_free_list():
    e, none = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 4, dtype=torch.int32, device="cuda")
    free = ints([1, 2, 7, 5, 3])
    for Lq in (0, 4, 5000):
        out = ints([-77])
        got = sa.pages_resize(e, none, e, free, ints([2]), 16, Lq, free_count_out=out)
        assert got[1] is out and out.item() == 2 and got[0].numel() == 0 and got[3].shape == (0, Lq)
        for count, want in ((-3, 0), (6, 5)):      # cut, and reported, as in a batch with sequences
            assert sa.pages_resize(e, none, e, free, ints([count]), 16, Lq, free_count_out=out)[1].item() == want
            refused()
    count = ints([2])
    sa.pages_resize(e, none, e, free, count, 16, 4, free_count_out=count)
    assert count.item() == 2 and free.tolist() == [1, 2, 7, 5, 3]
    sa.poll_status()


@pytest.mark.parametrize("units", [1, 2, 3, 5, 11, 100])
def test_means_of_the_smallest_numbers(units):
    # a mean of a few fp32 subnormal steps: the step of the mean's 8 bits is rounded so coarsely that the largest comes to more than 127 of them
    for d, block in ((64, 16), (128, 128)):
        K = torch.zeros(2, 128, 1, d, dtype=torch.bfloat16, device="cuda")
        K[1, 3, 0, 7], K[1, 5, 0, 11] = units * 2.0 ** -133, -units * 2.0 ** -133
        sums, scale = torch.full((2, 128 // block, 1, d), 9, dtype=torch.int8, device="cuda"), torch.full((2, 128 // block, 1), 7.0, device="cuda")
        sa.blocks_summarise(K, ints([[1]]), ints([128]), 128, sums, scale)
        sa.poll_status()
        mean = np.float32(units * 2.0 ** -133 / block)
        step = np.float32(mean * (np.float32(1) / np.float32(127)))
        q = min(127, int(np.rint(np.float32(mean / step))))
        assert scale[1, 0, 0].item() == step and sums[1, 0, 0, 7].item() == q and sums[1, 0, 0, 11].item() == -q
        assert sums[1, 0, 0].abs().sum().item() == 2 * q


def test_scales_an_eviction_cannot_use_are_refused():
    c = br.ScaledCache([200], 2, 64, 32, 16, seed=1, spare=5)
    dst = ints([c.spare[:3]])
    w = torch.rand(1, 2, c.max_pages * 32, device="cuda")
    k, v = c.scales["k_scale"], c.scales["v_scale"]
    call = lambda **kw: sa.kv_evict(w, c.K, c.V, dst_table=dst, sink=1, recent=30, heavy=40, **c.dev, **kw)
    before = [br.bits(x).clone() for x in (c.K, c.V)]
    for kw in (dict(v_scale=v), dict(k_scale=k), dict(k_scale=k[0], v_scale=v[0]), dict(k_scale=k[0, 0], v_scale=v), dict(k_scale=k, v_scale=v[0, 0]),
               dict(k_scale=k[0, 0].double(), v_scale=v[0, 0].double()), dict(k_scale=k[0, 0])):
        with pytest.raises(ValueError):
            call(**kw)
    assert all(torch.equal(br.bits(x), y) for x, y in zip((c.K, c.V), before))
    one = torch.ones(2, device="cuda")
    call(k_scale=one, v_scale=one)      # one to a head goes with every row: nothing to carry
    b = ref.Cache([200], 2, 64, 32, seed=1, spare=5)
    with pytest.raises(ValueError):
        sa.kv_evict(w, b.K, b.V, dst_table=ints([b.spare[:3]]), sink=1, recent=30, heavy=40, k_scale=one, v_scale=one, **b.dev)
    sa.poll_status()


def test_means_are_taken_anew_after_an_eviction():
    # the new pages' means are none of the old ones', and a choice goes by those of the rows that are there
    lens, Hkv, d, page, rows, block = [300, 260], 2, 64, 32, 16, 16
    budget, S, T, n = 160, 32, 8, 4
    need = -(-budget // page)
    c = br.ScaledCache(lens, Hkv, d, page, rows, seed=4, spare=2 * need)
    dst = ints(c.spare[:2 * need]).view(2, need)
    means = fresh_means(c, block)
    sa.blocks_summarise(c.K, c.dev["block_table"], c.dev["kv_len"], c.max_pages * page, *means, k_scale=c.scales["k_scale"])
    w = torch.rand(2, Hkv, c.max_pages * page, generator=torch.Generator().manual_seed(1)).cuda()
    _, kept, shift, _ = sa.kv_evict(w, c.K, c.V, dst_table=dst, sink=2, recent=60, heavy=budget - 62, **c.dev, **c.scales)
    assert (means[0][dst[0, 0].long()] == 9).all()      # as they were
    sa.blocks_summarise(c.K, dst, kept, need * page, *means, k_scale=c.scales["k_scale"])
    Q = rand(2, 1, 4, d)
    got = sa.blocks_select(Q, *means, dst, kept, page, S, T, n, head_past_mask=[1, 1], pos_shift=shift)
    sa.poll_status()
    c.table = dst.cpu()
    same_means(c, block, means, kept.tolist())
    for b in range(2):
        want = br.select(Q[b].float().cpu().double().numpy(), means[0].cpu().numpy(), means[1].cpu().numpy(), dst[b].tolist(), budget, 1, S, T, [1, 1], page, block, n, 0,
                         shift=int(shift[b]))
        assert np.array_equal(got[b].cpu().numpy(), want)


@pytest.mark.parametrize("Lq", [4, 3000])
def test_positions_past_their_type_are_refused(Lq):
    # a shift that brings a new row's position past 2^31 - 1 counts as one out of range: the sequence's positions are its slots
    page, top = 16, 2 ** 31 - 1
    lens, want = [40, 33, 7], [43, 33, 8]
    table = ints([[3 * b + i for i in range(3)] + [-1] * 300 for b in range(3)])
    for shift, bad in (([top - 42, top, 5], False), ([top - 41, 3, 5], True), ([top, 3, 5], True)):
        got = sa.pages_resize(ints(want), table.clone(), ints(lens), ints(list(range(20, 60))), ints([40]), page, Lq, pos_shift=ints(shift))
        refused() if bad else sa.poll_status()
        assert got[4][0, :4].tolist() == [(0 if bad else shift[0]) + 40 + t for t in range(3)] + [0]
        assert got[4][2, :2].tolist() == [12, 0] and got[4][1].eq(0).all() and got[0].tolist() == want


@pytest.mark.parametrize("top", [448 * 2.0 ** 119, 3.3895313892515355e38])
def test_the_largest_numbers_saturate(top):
    # scales end at 2^119: finite magnitudes past 448 * 2^119 (bf16 goes to 1.99 * 2^127) saturate like infinities
    c = br.ScaledCache([16], 1, 64, 16, 16, seed=1)
    K, V = torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16, device="cuda"), rand(1, 16, 1, 64)
    K[0, 3, 0, 5], K[0, 4, 0, 6] = top, -top
    assert K[0, 3, 0, 5].item() == top
    sa.kv_append(K, V, c.K, c.V, **c.dev, **c.scales)
    sa.poll_status()
    at = c.table[0, 0].long()
    x = c.K[at].float()
    assert c.scales["k_scale"][at, 0, 0].item() == 2.0 ** 119 and x[3, 0, 5].item() == 448 and x[4, 0, 6].item() == -448 and x.abs().sum().item() == 896
