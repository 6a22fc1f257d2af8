"""Scaled caches and chosen blocks where a thread block goes through many tiles and several items (rings that wrap, bases that move, parts
of items at both ends), against the definition in 64 bits on the device; many sequences read the same pages."""
import numpy as np
import pytest
import torch

import blocks_ref as br
import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def build(kind, d, Hkv, page, rows, n_pages, B, lens, seed, trend):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn(n_pages, page, Hkv, d, generator=g, device="cuda") for _ in range(2))
    per = max(-(-n // page) for n in lens)
    table = torch.stack([torch.randperm(n_pages, generator=g, device="cuda")[:per] for _ in range(B)]).int()
    if trend:      # keys grow along the first sequence: its rows' bases move again and again, up or down the list
        order = table[0].long()
        k[order] *= torch.linspace(0.2, 3, per, device="cuda")[:, None, None, None]
    scales = {}
    if kind == "bf16":
        K, V = k.bfloat16(), v.bfloat16()
    else:
        K, V = ((60 * x).clamp(-448, 448).to(E4M3) for x in (k, v))
        shape = (Hkv,) if kind == "heads" else (n_pages, page // rows, Hkv)
        scales = {x: torch.exp2(torch.randint(-8, -3, shape, generator=g, device="cuda").float()) for x in ("k_scale", "v_scale")}
        if kind == "odd":      # no powers of two
            scales = {x: s * (1 + torch.rand(shape, generator=g, device="cuda")) for x, s in scales.items()}
    return K, V, table, scales


def exact(Q, K, V, scales, table, n, q, S, T, mask, idx, block, page, b):
    """O, LSE and the bound's parts of sequence b's new rows, in 64 bits: [q, Hq, d], [Hq, q], ..."""
    Hkv, d = K.shape[2:]
    g = Q.shape[2] // Hkv
    O, spread = np.zeros((q, Hkv * g, d)), np.zeros((q, Hkv * g, d))
    lse, terms = np.zeros((Hkv * g, q)), np.zeros((Hkv * g, q))
    for t in range(q):
        for h in range(Hkv):
            j = br.visible(n, q, t, mask[h], S, T, 0, None if idx is None else idx[b, t, h].tolist(), block)
            j = torch.from_numpy(j).cuda()
            at = table[b, j // page].long(), j % page
            k, v = (x.view(torch.uint8)[at[0], at[1], h].view(x.dtype).double() if x.dtype == E4M3 else x[at[0], at[1], h].double() for x in (K, V))
            vs = None
            if scales:
                ks, vs = ((s[h].double().expand(len(j)) if s.dim() == 1 else s[at[0], at[1] // (page // s.shape[1]), h].double())
                          for s in (scales["k_scale"], scales["v_scale"]))
                k, v = k * ks[:, None], v * vs[:, None]
            qq = Q[b, t, h * g:(h + 1) * g].double()
            x = qq @ k.T * d ** -0.5
            p = torch.softmax(x, -1)
            sp = p @ v.abs()
            if vs is not None:      # fp16's step below its normal range, as in blocks_ref.attend
                sp += 2.0 ** -37 / ref.FP16 * (p * vs).amax(-1, keepdim=True) * (v.abs() / vs[:, None]).sum(0)
            rows = slice(h * g, (h + 1) * g)
            O[t, rows], spread[t, rows], lse[rows, t] = (p @ v).cpu(), sp.cpu(), torch.logsumexp(x, -1).cpu()
            terms[rows, t] = (qq.abs() @ k.abs().T).amax(-1).cpu() * d ** -0.5
    return O, lse, spread, terms


def run(kind, d, Hkv, g, Lq, page, rows, B, hi, S, T, mask, n, block, seed, trend=False):
    r = np.random.default_rng(seed)
    lens = [hi - int(r.integers(0, hi // 3)) for _ in range(B)]
    lens[0] = hi
    K, V, table, scales = build(kind, d, Hkv, page, rows, -(-hi // page) + 40, B, lens, seed, trend)
    Q = torch.randn(B, Lq, Hkv * g, d, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda").bfloat16()
    idx, kw = None, {}
    if n:
        idx = np.full((B, Lq, Hkv, n), -1, np.int32)
        for b in range(B):
            for t in range(Lq):
                room = br.first_whole(lens[b] - Lq + t, S, T, 0, block) // block
                for h in range(Hkv):
                    k = np.sort(r.permutation(room)[:n])
                    idx[b, t, h, :len(k)] = k
        kw = dict(blocks=torch.from_numpy(idx).cuda(), block=block)
    call = lambda: sa.seg_attn_decode(Q, K, V, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), S, T, mask, **scales, **kw)
    O, lse = call()
    O2, l2 = call()
    sa.poll_status()
    assert torch.equal(O, O2) and torch.equal(lse, l2)
    for b in (0, 1, B // 2, B - 1):
        want = exact(Q, K, V, scales, table, lens[b], Lq, S, T, mask, idx, block, page, b)
        ref.check_decode(O[b:b + 1], lse[b:b + 1], tuple(x[None] for x in want) + (None,), [Lq], d, fp8=bool(scales))


@pytest.mark.parametrize("trend", [False, True])
@pytest.mark.parametrize("kind", ["blocks", "odd"])
@pytest.mark.parametrize("d,g,Lq,page,rows", [(128, 4, 1, 64, 64), (128, 12, 1, 48, 16), (64, 4, 2, 128, 32), (64, 8, 2, 32, 32), (128, 4, 6, 64, 16), (128, 8, 8, 256, 128),
                                              (64, 4, 6, 64, 64), (64, 4, 16, 16, 16)])
def test_long_ranges_with_scales(d, g, Lq, page, rows, kind, trend):
    run(kind, d, 4, g, Lq, page, rows, 40, 5000, 1 << 30, 0, [1] * 4, 0, 0, seed=d + g + Lq, trend=trend)


@pytest.mark.parametrize("trend", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "heads", "blocks", "odd"])
@pytest.mark.parametrize("d,g,Lq,page,rows,block,n", [(128, 4, 1, 64, 64, 64, 60), (128, 12, 2, 48, 16, 16, 120), (64, 4, 3, 128, 32, 32, 100), (64, 16, 1, 32, 32, 32, 128),
                                                      (128, 20, 1, 128, 64, 128, 30)])
def test_long_ranges_of_chosen_blocks(d, g, Lq, page, rows, block, n, kind, trend):
    run(kind, d, 4, g, Lq, page, rows, 40, 9000, 700, 300, [1, 1, 0, 1], n, block, seed=d + g + n, trend=trend)


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_long_ranges_across_classes(kind):
    # eight heads of all classes, two to four of a class side by side
    run(kind, 128, 8, 4, 2, 64, 64, 48, 6000, 900, 200, [1, 0, 2, 1, 0, 1, 2, 1], 40, 64, seed=3)
    run(kind, 64, 8, 2, 1, 64, 64, 64, 6000, 900, 200, [1, 0, 1, 1, 0, 1, 0, 0], 40, 64, seed=4)
