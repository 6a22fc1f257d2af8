"""What the entry points for pages and blocks refuse before they touch a device, their structures, and the references themselves."""
import os
import subprocess

import numpy as np
import pytest
import torch

import blocks_ref as br
import paged_ref as ref
import paper_2605_11744_b200 as sa
from paper_2605_11744_b200 import blocks, paged
from test_paged_cpu import BAD_CACHES, ODD, OK, ST, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structures_are_packed_as_the_header_declares_them(tmp_path):
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "seg_attn.h"\nint main(void) {\n'
                   'printf("%zu %zu %zu %zu ", sizeof(seg_block_scales), offsetof(seg_block_scales, k_stride), offsetof(seg_block_scales, v_stride),'
                   ' offsetof(seg_block_scales, rows));\n'
                   'printf("%zu %zu %zu ", sizeof(seg_block_choice), offsetof(seg_block_choice, n), offsetof(seg_block_choice, block));\n'
                   'printf("%zu %zu\\n", sizeof(seg_block_means), offsetof(seg_block_means, block)); return 0; }\n')
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out == [paged._SCALES.size, 16, 40, 64, paged._CHOICE.size, 8, 12, blocks._MEANS.size, 16]


def scales(k=OK, v=OK, ks=(8, 2, 1), vs=(8, 2, 1), rows=16):
    return paged._SCALES.pack(k, v, *ks, *vs, rows)


def means(q=OK, scale=OK, block=16):
    return blocks._MEANS.pack(q, scale, block)


def choice(idx=OK, n=4, block=16):
    return paged._CHOICE.pack(idx, n, block)


def eight(**kw):
    return cache(dtype=1, **kw)


def decode(c, sc, ch, Lq=1, Hq=4, S=64, T=16, scale=0.1, mask=b"\0\1", Q=OK, qs=ST, O=OK, os_=ST, lse=OK, win=None, wout=None, W=0, ws=OK, ws_bytes=1 << 40):
    return sa.lib().seg_attn_decode_blocks(c, sc, ch, Lq, Hq, S, T, scale, mask + bytes(64), Q, qs, O, os_, lse, win, wout, W, ws, ws_bytes, None)


def append(c, sc, Lq=1, K=OK, ks=ST, V=OK, vs=ST, Hq=0, Q=None, qs=None, qo=None, qos=None, table=None, n_pos=0, rot=0, layout=0):
    return sa.lib().seg_blocks_append(c, sc, Lq, K, ks, V, vs, Hq, Q, qs, qo, qos, table, n_pos, rot, layout, None)


def summarise(c, sc, m, Lq=1):
    return sa.lib().seg_blocks_summarise(c, sc, Lq, m, None)


def select(c, m, Lq=1, Hq=4, S=64, T=16, mask=b"\0\1", Q=OK, qs=ST, n=4, sink=1, idx=OK):
    return sa.lib().seg_blocks_select(c, Lq, Hq, S, T, mask + bytes(64), Q, qs, m, n, sink, idx, None)


def evict(c, sc, w=OK, W=128, sink=1, recent=20, heavy=10, dst=OK, pages=2, stride=2, idx=OK << 3, n=OK, s=OK, wo=OK << 4):
    return sa.lib().seg_blocks_evict(c, sc, w, W, sink, recent, heavy, dst, pages, stride, idx, n, s, wo, None)


def resize(B=2, Lq=4, page=16, n_pages=40, want=OK, table=OK, per=8, stride=8, n=OK, shift=None, free=OK, count=OK, n_out=OK, c_out=OK, q=OK, slots=OK,
           pos=OK, ws=OK, ws_bytes=1 << 30):
    return sa.lib().seg_pages_resize(B, Lq, page, n_pages, want, table, per, stride, n, shift, free, count, n_out, c_out, q, slots, pos, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(bad):
    L = sa.lib()
    if "dtype" not in bad:
        c = eight(**bad)
        assert decode(c, scales(), None) == 1 and append(c, scales()) == 1 and evict(c, scales()) == 1 and L.seg_attn_decode_blocks_workspace_bytes(c, scales(), None, 1, 4, 0) == 0
        if "v_stride" not in bad and bad != dict(V=OK + 8):      # a summary reads keys alone
            assert summarise(c, scales(), means()) == 1
    c = cache(**bad)
    assert decode(c, None, choice()) == 1 and L.seg_attn_decode_blocks_workspace_bytes(c, None, choice(), 1, 4, 0) == 0
    if not set(bad) & {"dtype", "K", "V", "k_stride", "v_stride", "k_scale"}:      # a choice reads no values
        assert select(c, means()) == 1


@pytest.mark.parametrize("bad", [dict(k=0), dict(v=0), dict(k=OK + 2), dict(v=OK + 1), dict(ks=(-8, 2, 1)), dict(vs=(8, 2, -1)), dict(rows=0), dict(rows=8),
                                 dict(rows=32), dict(rows=48), dict(rows=256)], ids=str)
def test_bad_scales_are_refused(bad):
    assert decode(eight(), scales(**bad), None) == 1 and append(eight(), scales(**bad)) == 1 and evict(eight(), scales(**bad)) == 1
    if "v" not in bad and "vs" not in bad:
        assert summarise(eight(), scales(**bad), means()) == 1


def test_scales_of_blocks_belong_to_an_8_bit_cache_without_others():
    for c in (cache(), cache(dtype=1, k_scale=OK, v_scale=OK), cache(dtype=1, k_scale=OK)):
        assert decode(c, scales(), None) == 1 and append(c, scales()) == 1 and summarise(c, scales(), means()) == 1
    assert append(eight(), None) == 1 and decode(eight(), None, None) == 1 and evict(eight(), None) == 1


@pytest.mark.parametrize("bad", [dict(ks=(0, 2, 1)), dict(ks=(8, 2, 0)), dict(vs=(8, 0, 1))], ids=str)
def test_scales_that_are_written_are_apart(bad):
    c = eight(page_size=32)
    assert append(c, scales(**bad)) == 1 and evict(c, scales(**bad)) == 1
    assert decode(c, scales(**bad), None, ws=None) == 5      # reading them is fine


@pytest.mark.parametrize("bad", [dict(w=None), dict(W=127), dict(sink=-1), dict(sink=0, recent=0, heavy=0), dict(heavy=12), dict(dst=None), dict(stride=1),
                                 dict(idx=None), dict(n=None), dict(wo=OK), dict(idx=OK)], ids=str)
def test_bad_evictions_are_refused(bad):
    assert evict(eight(), scales(), **bad) == 1


@pytest.mark.parametrize("bad", [dict(idx=0), dict(idx=OK + 2), dict(n=0), dict(n=129), dict(n=-1), dict(block=0), dict(block=8), dict(block=32), dict(block=48)],
                         ids=str)
def test_bad_choices_are_refused(bad):
    assert decode(cache(), None, choice(**bad)) == 1 and decode(eight(), scales(), choice(**bad)) == 1


@pytest.mark.parametrize("bad", [dict(Lq=-1), dict(Hq=3), dict(Hq=0), dict(S=0), dict(T=-1), dict(T=65), dict(scale=0.0), dict(mask=b"\0\3"), dict(Q=None),
                                 dict(O=OK + 8), dict(lse=None), dict(qs=ODD), dict(os_=None), dict(wout=OK << 8, W=128), dict(Lq=1 << 28, Hq=64)], ids=str)
def test_bad_decode_calls_are_refused(bad):
    assert decode(cache(), None, choice(), **bad) == 1
    if "W" not in bad:
        assert decode(eight(), scales(), None, **bad) == 1
    assert decode(cache(), None, choice(), ws=None) == 5 and decode(eight(), scales(), None, ws=OK + 16) == 5
    assert decode(eight(), scales(), choice(), ws_bytes=16) == 5


@pytest.mark.parametrize("bad", [dict(Lq=-1), dict(K=None), dict(V=OK + 4), dict(ks=ODD), dict(vs=None), dict(Hq=4, Q=OK, qs=ST, qo=OK, qos=ST),
                                 dict(table=OK, n_pos=10, rot=24), dict(table=OK + 8, n_pos=10, rot=64), dict(table=OK, n_pos=10, rot=64, layout=2),
                                 dict(table=OK, n_pos=10, rot=64, Hq=4, Q=OK, qs=ST), dict(table=OK, n_pos=10, rot=64, Hq=0, Q=OK, qs=ST, qo=OK, qos=ST)],
                         ids=str)
def test_bad_append_calls_are_refused(bad):
    assert append(eight(), scales(), **bad) == 1


def test_appends_past_the_limits_are_refused():
    big = 0x7fffffff
    for B, Lq in ((1 << 15, 1 << 16), (65536, 1), (65535, big)):
        assert append(eight(B=B), scales(), Lq=Lq) == 1, (B, Lq)
    wide = eight(B=65535, Hkv=64, max_pages=1 << 18, table_stride=1 << 18)
    assert append(wide, scales(), Lq=1 << 15) == 1      # B * blocks * heads of units
    assert append(eight(), scales(), Lq=1 << 20, Hq=1 << 16, Q=OK, qs=ST, qo=OK, qos=ST, table=OK, n_pos=10, rot=64) == 1


@pytest.mark.parametrize("bad", [dict(q=0), dict(q=OK + 8), dict(scale=0), dict(scale=OK + 2), dict(block=0), dict(block=8), dict(block=32), dict(block=48)], ids=str)
def test_bad_means_are_refused(bad):
    assert summarise(cache(), None, means(**bad)) == 1 and select(cache(), means(**bad)) == 1


@pytest.mark.parametrize("bad", [dict(Lq=-1), dict(Hq=3), dict(Hq=0), dict(S=0), dict(T=-1), dict(T=65), dict(mask=b"\0\3"), dict(Q=None), dict(Q=OK + 2), dict(qs=ODD),
                                 dict(qs=None), dict(n=0), dict(n=129), dict(sink=-1), dict(sink=5), dict(idx=None), dict(idx=OK + 2)], ids=str)
def test_bad_selections_are_refused(bad):
    assert select(cache(), means(), **bad) == 1


def test_selections_past_the_limits_are_refused():
    assert select(cache(max_pages=1 << 19, table_stride=1 << 19), means()) == 1      # 2^19 blocks of 16
    assert select(cache(B=1 << 15), means(), Lq=1 << 15) == 1
    assert summarise(cache(), None, means(), Lq=-1) == 1 and summarise(None, None, means()) == 1 and select(None, means()) == 1
    assert summarise(cache(B=65535, Hkv=64, max_pages=1 << 16, table_stride=1 << 16), None, means(), Lq=1 << 20) == 1


@pytest.mark.parametrize("bad", [dict(B=-1), dict(B=65536), dict(Lq=-1), dict(page=0), dict(n_pages=-1), dict(per=-1), dict(stride=7),
                                 dict(per=1 << 27, stride=1 << 27), dict(want=None), dict(table=None), dict(n=None), dict(free=None), dict(count=None),
                                 dict(n_out=None), dict(c_out=None), dict(q=None), dict(slots=None), dict(slots=OK + 4), dict(pos=None)], ids=str)
def test_bad_resizes_are_refused(bad):
    assert resize(**bad) == 1
    for kw in (dict(ws=None), dict(ws=OK + 16), dict(ws_bytes=8)):
        assert resize(Lq=2049, **kw) == 5 and resize(B=1025, Lq=1, **kw) == 5
    L = sa.lib()
    assert L.seg_pages_workspace_bytes(-1) == 0 and L.seg_pages_workspace_bytes(65536) == 0 and L.seg_pages_workspace_bytes(0) > 0


def test_nothing_to_do_is_fine_without_a_device():
    assert evict(eight(B=0), scales()) == 0
    assert resize(B=0) == 0 and append(eight(B=0), scales()) == 0 and append(eight(), scales(), Lq=0) == 0
    assert decode(eight(B=0), scales(), None) == 0 and decode(cache(), None, choice(), Lq=0) == 0
    assert summarise(cache(B=0), None, means()) == 0 and summarise(cache(), None, means(), Lq=0) == 0 and summarise(cache(n_pages=0), None, means()) == 0
    assert select(cache(B=0), means()) == 0 and select(cache(), means(), Lq=0) == 0


def test_no_device_means_an_error_not_a_fallback():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert resize() in (2, 3) and append(eight(), scales()) in (2, 3) and decode(eight(), scales(), None) in (2, 3)
    assert decode(cache(), None, choice()) in (2, 3) and summarise(cache(), None, means()) in (2, 3) and select(cache(), means()) in (2, 3)


def test_wrappers_refuse_what_is_not_a_cache():
    K = torch.zeros(4, 32, 2, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    sums, sc = torch.zeros(4, 2, 2, 64, dtype=torch.int8), torch.zeros(4, 2, 2)
    with pytest.raises(ValueError, match="CUDA"):
        sa.blocks_summarise(K, t, n, 1, sums, sc)
    with pytest.raises(ValueError, match="CUDA|contiguous"):
        sa.blocks_select(torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), sums, sc, t, n, 32, 64, 16, 4)
    with pytest.raises(ValueError, match="CUDA"):
        sa.pages_resize(n, t, n, n, n, 16, 1)
    with pytest.raises(ValueError, match="8-bit"):
        paged._block_scales(sc, sc, K, -1)
    with pytest.raises(ValueError, match="8-bit"):
        paged._block_scales(torch.zeros(4, 3, 2), torch.zeros(4, 3, 2), K.to(torch.float8_e4m3fn), -1)
    with pytest.raises(ValueError, match="v_scale"):
        paged._block_scales(sc, None, K.to(torch.float8_e4m3fn), -1)


# ---- the references themselves ------------------------------------------------------------------------------------------

def test_reference_pages_are_conserved():
    rng = np.random.default_rng(3)
    for trial in range(200):
        B, page, per = int(rng.integers(1, 9)), int(rng.integers(1, 9)), 6
        n_pages = B * per - int(rng.integers(0, 5))
        order = rng.permutation(n_pages).tolist()
        lens, table = [], []
        for b in range(B):
            n = int(rng.integers(0, min(per * page, len(order) * page // B + 1) + 1))
            k = min(-(-n // page), len(order))
            lens.append(min(n, k * page))
            table.append([order.pop() for _ in range(k)] + [-1] * (per - k))
        want = [int(rng.integers(0, per * page + 1)) for _ in range(B)]
        t, n, free, q, slots, pos = br.resize(want, table, lens, order, len(order), page, 5)
        held = [t[b][k] for b in range(B) for k in range(-(-n[b] // page))] + free
        assert sorted(held) == list(range(n_pages))
        for b in range(B):
            assert n[b] in (want[b], lens[b]) and q[b] == max(0, n[b] - lens[b]) <= 5
            assert [s for s in slots[b] if s >= 0] == [t[b][(lens[b] + i) // page] * page + (lens[b] + i) % page for i in range(q[b])]


def test_reference_scales_are_the_smallest_that_fit():
    for x in (1.0, 448.0, 448.0001, 447.9, 3.5, 1e-5, 2.0 ** -31 * 1.75, 1e30):
        s = br.scale_of(np.float32(x))
        assert np.float32(x) <= 448 * s and (np.float32(x) > 448 * s / 2 or s == 2.0 ** -40)
    assert br.scale_of(0.0) == 2.0 ** -40 and br.scale_of(3e38) == 2.0 ** 119


def test_reference_attention_over_all_blocks_is_the_whole_past():
    rng = np.random.default_rng(1)
    n, Hkv, d, page, block, S, T = 200, 2, 64, 32, 16, 32, 8
    K, V, Q = rng.standard_normal((7, page, Hkv, d)), rng.standard_normal((7, page, Hkv, d)), rng.standard_normal((1, 3, 4, d))
    table = rng.permutation(7)[None]
    idx = np.full((1, 3, Hkv, 13), -1)
    for t in range(3):
        room = br.first_whole(n - 3 + t, S, T, 0, block) // block
        idx[0, t, :, :room] = np.arange(room)
    a = br.attend(Q, K, V, table, [n], [3], S, T, [1, 0], 0.1, page, idx=idx, block=block, cap=224)
    b = ref.decode(Q, K, V, table, [n], [3], S, T, [1, 0], 0.1, page)
    for x, y in zip(a, b):
        assert np.allclose(x, y, atol=1e-12)
