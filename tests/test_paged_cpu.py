"""What the paged cache's entry points refuse before they touch a device, the layout of their structures, and the references
themselves against an independent statement of the mask."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import oracle
import paged_ref as ref
import paper_2605_11744_b200 as sa
from paper_2605_11744_b200 import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = 1 << 20      # a 256-byte aligned address that nothing reads: every refusal comes before the first launch


def test_library_exports_the_paged_entry_points():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "seg_attn.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(seg_kv_[a-z_]+)\s*\(", text)))
    assert names == ["seg_kv_append", "seg_kv_evict"]
    for n in names + ["seg_attn_decode", "seg_rope_rotate", "seg_rope_table_scaled"]:
        assert hasattr(sa.lib(), n), n


def test_structures_are_packed_as_the_header_declares_them(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "seg_attn.h"\nint main(void) {\n'
                   'printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(seg_kv_cache), offsetof(seg_kv_cache, K), offsetof(seg_kv_cache, k_stride),'
                   ' offsetof(seg_kv_cache, k_scale), offsetof(seg_kv_cache, pos_shift), offsetof(seg_rope_scaling, base));\n'
                   'printf("%zu\\n", sizeof(seg_rope_scaling)); return 0; }\n')
    exe = tmp_path / "s"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out[0] == paged._CACHE.size and out[1:6] == [32, 48, 96, 136, 8] and out[6] == paged._SCALING.size


def cache(**kw):
    f = dict(B=2, Hkv=2, d=128, dtype=0, page_size=16, n_pages=40, max_pages=8, table_stride=8, K=OK, V=OK, k_stride=(4096, 256, 128),
             v_stride=(4096, 256, 128), k_scale=0, v_scale=0, block_table=OK, kv_len=OK, q_len=0, pos_shift=0)
    f.update(kw)
    return paged._CACHE.pack(f["B"], f["Hkv"], f["d"], f["dtype"], f["page_size"], f["n_pages"], f["max_pages"], f["table_stride"], f["K"],
                             f["V"], *f["k_stride"], *f["v_stride"], f["k_scale"], f["v_scale"], f["block_table"], f["kv_len"],
                             f["q_len"], f["pos_shift"])


BAD_CACHES = [dict(B=-1), dict(Hkv=0), dict(Hkv=65), dict(d=96), dict(dtype=2), dict(page_size=0), dict(n_pages=-1), dict(max_pages=-1),
              dict(table_stride=7), dict(max_pages=1 << 27, table_stride=1 << 27), dict(K=0), dict(V=OK + 8), dict(k_stride=(4096, 256, 124)),
              dict(v_stride=(-4096, 256, 128)), dict(k_scale=OK), dict(dtype=1), dict(dtype=1, k_scale=OK, v_scale=OK, k_stride=(4096, 256, 136)),
              dict(block_table=0), dict(kv_len=0)]
ST = paged._STRIDE3.pack(1024, 512, 128)
ODD = paged._STRIDE3.pack(1024, 512, 124)


def decode(c, Lq=1, Hq=4, S=64, T=16, scale=0.1, mask=b"\0\1", Q=OK, qs=ST, O=OK, os_=ST, lse=OK, win=None, wout=None, W=0, ws=OK,
           ws_bytes=1 << 40):
    return sa.lib().seg_attn_decode(c, Lq, Hq, S, T, scale, ctypes.create_string_buffer(mask, 64), Q, qs, O, os_, lse, win, wout, W, ws,
                                    ws_bytes, None)


def append(c, Lq=1, K=OK, ks=ST, V=OK, vs=ST, Hq=0, Q=None, qs=None, qo=None, qos=None, table=None, n_pos=0, rot=0, layout=0):
    return sa.lib().seg_kv_append(c, Lq, K, ks, V, vs, Hq, Q, qs, qo, qos, table, n_pos, rot, layout, None)


def evict(c, w=OK, W=128, sink=1, recent=20, heavy=10, dst=OK, pages=2, stride=2, idx=OK << 3, n=OK, s=OK, wo=OK << 4):
    return sa.lib().seg_kv_evict(c, w, W, sink, recent, heavy, dst, pages, stride, idx, n, s, wo, None)


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(bad):
    c = cache(**bad)
    assert decode(c) == 1 and append(c) == 1 and sa.lib().seg_attn_decode_workspace_bytes(c, 1, 4, 0) == 0
    if bad != dict(dtype=1):      # without scales: an eviction reads no values
        assert evict(c) == 1


@pytest.mark.parametrize("bad", [dict(Lq=-1), dict(Hq=3), dict(Hq=0), dict(S=0), dict(T=-1), dict(T=65), dict(scale=0.0), dict(scale=float("nan")),
                                 dict(mask=b"\0\3"), dict(Q=None), dict(Q=OK + 2), dict(O=OK + 8), dict(lse=None), dict(lse=OK + 2), dict(qs=ODD),
                                 dict(os_=None), dict(win=OK), dict(wout=OK, W=127), dict(wout=OK, win=OK + 64, W=128)], ids=str)
def test_bad_decode_calls_are_refused(bad):
    assert decode(cache(), **bad) == 1


def units(at, strides, shape, d):
    # the 16-byte pieces that a tensor of 16-bit elements covers
    rows = [at // 16 + (i * strides[0] + j * strides[1] + k * strides[2]) // 8 for i in range(shape[0]) for j in range(shape[1]) for k in range(shape[2])]
    return {r + x for r in rows for x in range(d // 8)}


def test_outputs_that_share_elements_with_the_queries_are_refused():
    # Without a workspace a call that passes comes to 5 before it touches a device.  Against the sets of elements themselves:
    # nested strides, permuted ones, expanded ones, interleaved views, unequal strides
    rng = np.random.default_rng(5)
    seen = [0, 0]
    for trial in range(1500):
        B, Lq, Hq, d = int(rng.integers(1, 4)), int(rng.integers(1, 5)), 2 * int(rng.integers(1, 4)), 64
        kind = trial % 5
        order = rng.permutation(3)
        def nest(gap):
            s, size = [0, 0, 0], d
            for i in order:
                s[i] = size + 8 * int(rng.integers(0, gap + 1))
                size = s[i] * (B, Lq, Hq)[i]
            return s
        qs = nest(12)
        os_ = list(qs) if kind < 3 else nest(12)
        if kind == 2:
            qs[int(rng.integers(0, 3))] = 0
        if kind == 4:
            qs, os_ = [8 * int(x) for x in rng.integers(0, 60, 3)], [8 * int(x) for x in rng.integers(0, 60, 3)]
        span = sum(s * (n - 1) for s, n in zip(qs, (B, Lq, Hq))) + d
        at = OK + 2 * 8 * int(rng.integers(-span // 8 - 2, span // 8 + 3))
        pack = lambda s: paged._STRIDE3.pack(*s)
        got = decode(cache(B=B, d=d), Lq=Lq, Hq=Hq, Q=OK, qs=pack(qs), O=at, os_=pack(os_), ws=None)
        same = at == OK and all(n == 1 or a == b for a, b, n in zip(qs, os_, (B, Lq, Hq)))
        shared = bool(units(OK, qs, (B, Lq, Hq), d) & units(at, os_, (B, Lq, Hq), d))
        assert got == (1 if shared and not same else 5), (trial, qs, os_, at - OK, (B, Lq, Hq))
        seen[shared] += 1
    assert min(seen) > 100      # both answers were asked for
    # queries and outputs side by side in one buffer, large; a row more would meet
    big = dict(Lq=4096, Hq=64, qs=paged._STRIDE3.pack(4096 * 128 * 128, 128 * 128, 128), os_=paged._STRIDE3.pack(4096 * 128 * 128, 128 * 128, 128), ws=None)
    assert decode(cache(), O=OK + 2 * 64 * 128, **big) == 5 and decode(cache(), O=OK + 2 * 63 * 128, **big) == 1
    # the same view, unless the weights of many rows read the queries again (a bf16 cache, from 33 rows to a KV head on)
    for Lq, kw, want in ((1, {}, 5), (8, dict(wout=OK << 8, W=128), 5), (16, {}, 5), (16, dict(wout=OK << 8, W=128), 5), (17, {}, 5),
                         (17, dict(wout=OK << 8, W=128), 1)):
        assert decode(cache(), Lq=Lq, Hq=4, ws=None, **kw) == want, (Lq, kw)
    eight = cache(dtype=1, k_scale=OK, v_scale=OK)
    assert decode(eight, Lq=17, Hq=4, ws=None, wout=OK << 8, W=128) == 5


def test_missing_workspaces_are_refused():
    for kw in (dict(ws=None), dict(ws=OK + 16), dict(ws_bytes=16)):
        assert decode(cache(), **kw) == 5


@pytest.mark.parametrize("bad", [dict(Lq=-1), dict(K=None), dict(V=OK + 4), dict(ks=ODD), dict(vs=None),
                                 dict(Hq=4, Q=OK, qs=ST, qo=OK, qos=ST),                                              # queries without a table
                                 dict(table=OK, n_pos=10, rot=130), dict(table=OK, n_pos=10, rot=24), dict(table=OK, n_pos=10, rot=0),
                                 dict(table=OK + 8, n_pos=10, rot=64), dict(table=OK, n_pos=10, rot=64, layout=2), dict(table=OK, n_pos=-1, rot=64),
                                 dict(table=OK, n_pos=10, rot=64, Hq=4, Q=OK, qs=ST), dict(table=OK, n_pos=10, rot=64, Hq=0, Q=OK, qs=ST, qo=OK, qos=ST),
                                 dict(table=OK, n_pos=10, rot=64, Hq=4, Q=OK, qs=ODD, qo=OK, qos=ST)], ids=str)
def test_bad_append_calls_are_refused(bad):
    assert append(cache(), **bad) == 1


@pytest.mark.parametrize("bad", [dict(w=None), dict(W=127), dict(sink=-1), dict(heavy=-1), dict(sink=0, recent=0, heavy=0), dict(heavy=12),
                                 dict(dst=None), dict(stride=1), dict(idx=None), dict(n=None), dict(s=None), dict(wo=None), dict(wo=OK),
                                 dict(wo=OK + 1024), dict(idx=OK), dict(sink=2000000000, recent=2000000000)], ids=str)
def test_bad_evictions_are_refused(bad):
    assert evict(cache(), **bad) == 1


def test_bad_rotations_are_refused():
    L = sa.lib()

    def rot(B=1, L_=2, H=4, d=128, r=128, lay=0, X=OK, xs=ST, Y=OK, ys=ST, pos=None, pos0=0, table=OK, n_pos=10):
        return L.seg_rope_rotate(B, L_, H, d, r, lay, X, xs, Y, ys, pos, pos0, 0, table, n_pos, None)
    for bad in (dict(B=-1), dict(L_=-1), dict(H=0), dict(d=72), dict(d=272, r=16), dict(r=8), dict(r=144), dict(r=20), dict(lay=2), dict(X=None),
                dict(Y=OK + 8), dict(xs=ODD), dict(ys=None), dict(pos0=-1), dict(pos0=9), dict(table=None), dict(table=OK + 4),
                dict(n_pos=(1 << 24) + 1)):
        assert rot(**bad) == 1, bad
    sc = lambda kind=0, base=1e4, factor=2.0, length=64.0, lo=1.0, hi=2.0, amp=1.0: paged._SCALING.pack(kind, base, factor, length, lo, hi, amp)
    for bad in (dict(kind=3), dict(base=1.0), dict(base=float("inf")), dict(amp=0.0), dict(kind=1, factor=0.0), dict(kind=2, factor=float("nan")),
                dict(kind=2, length=0.0), dict(kind=2, lo=-1.0), dict(kind=2, lo=2.0), dict(kind=2, hi=float("inf"))):
        assert L.seg_rope_table_scaled(8, 64, sc(**bad), OK, None) == 1, bad
    assert L.seg_rope_table_scaled(8, 60, sc(), OK, None) == 1 and L.seg_rope_table_scaled(-1, 64, sc(), OK, None) == 1
    assert L.seg_rope_table_scaled(8, 64, None, OK, None) == 1 and L.seg_rope_table_scaled(8, 64, sc(), None, None) == 1
    assert L.seg_rope_table_scaled(0, 64, sc(), None, None) == 0


def test_block_ranges_that_nobody_wrote_are_not_followed(tmp_path):
    # the join takes an item's first and last block from scratch memory, which after an expired wait holds anything
    src, exe = tmp_path / "parts.cu", tmp_path / "parts"
    src.write_text('#include <cstdio>\n#include <climits>\n#include "decode_kernels.cuh"\nint main() {\n'
                   'const int blocks = 148, v[] = {INT_MIN, -5, -1, 0, 1, 3, 147, 148, 160, 0x5a5a5a5a, INT_MAX};\n'
                   'for (int a : v) for (int b : v) {\n'
                   '  const bool parts = 0 <= a && a < blocks && 0 <= b && b < blocks && a < b;\n'
                   '  if (segattn::parts_to_join(a, b, blocks) != parts) { printf("%d %d\\n", a, b); return 1; }\n'
                   '}\nstatic_assert(segattn::kDecMaxBlocks >= 160, "room for the weights of every part");\nreturn 0; }\n')
    csrc = os.path.join(ROOT, "paper_2605_11744_b200", "csrc")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", csrc, "-I", os.path.join(ROOT, "include"),
                           "-o", str(exe), str(src)])
    assert subprocess.run([str(exe)]).returncode == 0
    text = open(os.path.join(csrc, "decode_kernels.cuh")).read()
    assert re.search(r"item_blocks\[blockIdx\.x\];\s*if \(!parts_to_join\(blocks\.x, blocks\.y, p\.blocks\)\) return;", text)


def test_rotations_and_appends_past_the_limits_are_refused():
    big = 0x7fffffff
    for B, n, H in ((1 << 16, 1 << 15, 1), (big, big, 1), (big, big, big), (1, 1, big), (1, 1 << 20, 1 << 14), (2, 1 << 24, 511)):
        assert sa.lib().seg_rope_rotate(B, n, H, 128, 128, 0, OK, ST, OK, ST, OK, 0, 0, OK, 10, None) == 1, (B, n, H)
    for B, Lq, Hq in ((1 << 15, 1 << 16, 0), (65535, big, 0), (1, 1 << 20, 1 << 14), (1, big, big)):
        kw = dict(Hq=Hq, Q=OK, qs=ST, qo=OK, qos=ST, table=OK, n_pos=10, rot=64) if Hq else {}
        assert append(cache(B=B), Lq=Lq, **kw) == 1, (B, Lq, Hq)


def test_nothing_to_do_is_fine_without_a_device():
    assert decode(cache(B=0)) == 0 and append(cache(B=0)) == 0 and evict(cache(B=0)) == 0
    assert decode(cache(), Lq=0) == 0 and append(cache(), Lq=0) == 0
    assert sa.lib().seg_rope_rotate(0, 5, 1, 64, 64, 0, None, None, None, None, None, 0, 0, None, 8, None) == 0


def test_no_device_means_an_error_not_a_fallback():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert decode(cache()) in (2, 3) and append(cache()) in (2, 3) and evict(cache()) in (2, 3)


def test_wrappers_refuse_what_is_not_a_cache():
    K = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        sa.seg_attn_decode(torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), K, K, t, n, 64, 16)
    with pytest.raises(ValueError, match="CUDA"):
        sa.kv_append(K[:1, :1], K[:1, :1], K, K, t, n)
    with pytest.raises(ValueError, match="CUDA"):
        sa.kv_evict(torch.zeros(1, 2, 32), K, K, t, n, t, 0, 1, 1)
    with pytest.raises(ValueError, match="CUDA"):
        sa.rope_rotate(K, torch.zeros(8, 32, 2))
    with pytest.raises(ValueError, match="kind"):
        sa.rope_table_scaled(8, 64, kind="none", device="cpu")


def test_reference_decode_is_the_last_row_of_the_segment_attention():
    # the reference of the GPU tests against the framework's own oracle, cut from a whole sequence
    rng = np.random.default_rng(0)
    n, Hq, Hkv, d, S, T, page = 90, 6, 3, 64, 32, 8, 16
    mask = [0, 1, 2]
    Q, K, V = rng.standard_normal((1, n, Hq, d)), rng.standard_normal((1, n, Hkv, d)), rng.standard_normal((1, n, Hkv, d))
    O, LSE = oracle.fwd(Q, K, V, S, T, mask)
    perm = rng.permutation(6)
    pad = np.zeros((1, 96 - n, Hkv, d))
    pages = lambda x: np.concatenate([x, pad], 1)[0].reshape(6, page, Hkv, d)[np.argsort(perm)]
    got = ref.decode(Q[:, -5:], pages(K), pages(V), perm[None], [n], [5], S, T, mask, d ** -0.5, page)
    assert np.abs(got[0] - O[:, -5:]).max() < 1e-12 and np.abs(got[1] - LSE[:, :, -5:]).max() < 1e-12
    assert abs(got[4].sum() - 5 * Hq) < 1e-9


def test_reference_rotation_is_the_oracle_s():
    from oracle import rope
    x = np.random.default_rng(1).standard_normal((1, 9, 2, 64))
    w = ref.frequencies(64)
    a = np.arange(9)[:, None] * w[None]
    tab = np.stack([np.cos(a), np.sin(a)], -1)[None]
    assert np.abs(ref.rotate(x, tab, "half") - rope.rotate(x, np.arange(9))).max() < 1e-12
    assert np.abs(ref.rotate(ref.rotate(x, tab, "interleaved"), tab, "interleaved", inverse=True) - x).max() < 1e-12
