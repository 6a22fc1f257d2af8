"""Rotary positions in general form against 64-bit arithmetic: scaled tables, both pairings, part of the head, given positions,
and the transposed map as the gradient."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2605_11744_b200 as sa

pytestmark = pytest.mark.gpu


def f64(t):
    return t.float().cpu().double().numpy()


@pytest.mark.parametrize("kw", [
    dict(),
    dict(base=500000.0, amplitude=0.75),
    dict(kind="linear", factor=4.0),
    dict(kind="by_parts", factor=8.0, trained_len=8192.0, turns_lo=1.0, turns_hi=32.0, amplitude=1.2),
    dict(kind="by_parts", factor=2.5, trained_len=64.0, turns_lo=0.0, turns_hi=0.5),
])
@pytest.mark.parametrize("n_pos,rot", [(1, 16), (1000, 96), (70000, 128), (300, 256)])
def test_scaled_tables(n_pos, rot, kw):
    t = sa.rope_table_scaled(n_pos, rot, **kw).cpu().numpy().astype(np.float64)
    kw = dict(kw)
    amp = kw.pop("amplitude", 1.0)
    a = np.arange(n_pos)[:, None] * ref.frequencies(rot, **kw)[None]
    # one rounding to fp32; the double angles of two evaluations differ by a few 2^-53 of angles up to 7e4
    assert np.abs(t[..., 0] - amp * np.cos(a)).max() <= amp * (ref.FP32 + 1e-10)
    assert np.abs(t[..., 1] - amp * np.sin(a)).max() <= amp * (ref.FP32 + 1e-10)


def test_plain_scaled_table_is_the_framework_s_own():
    assert torch.equal(sa.rope_table_scaled(777, 128, 10000.0), sa.rope_table(777, 128, 10000.0))


CASES = [(1, 1, 1, 64, 64), (2, 300, 5, 128, 128), (3, 7, 32, 128, 32), (1, 129, 3, 80, 48), (1, 40, 2, 256, 256), (2, 33, 9, 96, 16),
         (1, 2000, 32, 128, 96)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,L,H,d,rot", CASES)
def test_rotation_and_its_transpose(B, L, H, d, rot, layout):
    g = torch.Generator().manual_seed(L)
    X = torch.randn(B, L, H + 1, d, generator=g).bfloat16().cuda()[:, :, :H]
    table = sa.rope_table_scaled(L + 500, rot, amplitude=1.5)
    pos = torch.randint(0, L + 500, (B, L), generator=g, dtype=torch.int32)
    tab = table.cpu().numpy()
    for inverse in (False, True):
        for positions in (pos, None):
            Y = sa.rope_rotate(X, table, positions=None if positions is None else positions.cuda(), pos0=17, layout=layout, inverse=inverse)
            rows = tab[pos.numpy()] if positions is not None else np.broadcast_to(tab[17:17 + L], (B, L) + tab.shape[1:])
            want = ref.rotate(f64(X), rows.astype(np.float64), layout, inverse)
            # two products of at most 1.5 |x| and a sum, each rounded to fp32, and one rounding to bf16
            slack = 8 * ref.FP32 * 1.5 * np.abs(f64(X)).max(-1, keepdims=True)
            assert (np.abs(f64(Y) - want) <= ref.BF16 * np.abs(want) + slack).all()
            assert torch.equal(Y[..., rot:], X[..., rot:])
            # operation by operation in fp32: the same bits
            same = torch.from_numpy(ref.rotate(X.float().cpu().numpy(), rows, layout, inverse)).bfloat16()
            assert torch.equal(Y.cpu(), same)
    sa.poll_status()
    Z = X.clone()
    assert sa.rope_rotate(Z, table, pos0=17, layout=layout, out=Z) is Z
    assert torch.equal(Z, sa.rope_rotate(X, table, pos0=17, layout=layout))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_the_transpose_is_the_gradient(layout):
    # <dY, Rot X> against central differences of the 64-bit rotation, and against autograd through it
    B, L, H, d, rot = 1, 5, 2, 64, 48
    g = torch.Generator().manual_seed(3)
    X, dY = torch.randn(B, L, H, d, generator=g).bfloat16().cuda(), torch.randn(B, L, H, d, generator=g).bfloat16().cuda()
    table = sa.rope_table_scaled(L, rot, kind="linear", factor=2.0, amplitude=1.1)
    dX = f64(sa.rope_rotate(dY, table, layout=layout, inverse=True))
    tab = table.cpu().numpy().astype(np.float64)[None]
    x, dy = f64(X), f64(dY)
    f = lambda v: float((ref.rotate(v, tab, layout) * dy).sum())
    rng = np.random.default_rng(0)
    for _ in range(40):
        at = tuple(rng.integers(0, n) for n in x.shape)
        e = np.zeros_like(x)
        e[at] = 0.5
        diff = f(x + e) - f(x - e)       # the map is linear: exact up to round-off
        assert abs(diff - dX[at]) <= ref.BF16 * abs(diff) + 1e-5


def test_a_position_out_of_the_table_is_reported():
    X = torch.ones(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    table = sa.rope_table_scaled(10, 32)
    Y = sa.rope_rotate(X, table, positions=torch.tensor([[0, 10, -1, 9]], dtype=torch.int32, device="cuda"))
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 1
    assert torch.equal(Y[0, 0], X[0, 0]) and not Y[0, 1:3].any() and Y[0, 3].any()
    with pytest.raises(sa.SegAttnError):
        sa.rope_rotate(X, table, pos0=7)
    sa.poll_status()


def test_a_refused_input_does_not_end_the_waits_of_other_kernels():
    # until it is polled, a refused position stays in the status that all kernels share: a wait goes on to its own limit all
    # the same (1 ms here), and what that reports is the graver of the two; after the poll it is clear
    X = torch.ones(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    table = sa.rope_table_scaled(10, 32)
    bad = torch.tensor([[0, 10, -1, 9]], dtype=torch.int32, device="cuda")
    sa.rope_rotate(X, table, positions=bad)
    sa.selftest_wait_timeout()
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 4
    sa.poll_status()
    sa.selftest_wait_timeout()          # the other way round
    sa.rope_rotate(X, table, positions=bad)
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 4
    # a training step with a refused input outstanding is the step it would have been
    from util import rand_inputs
    Q, K, V, dO = rand_inputs(1, 1500, 4, 2, 128, seed=4)
    O, lse = sa.seg_attn_fwd(Q, K, V, 256, 64, [0, 1])
    want = (O, lse) + tuple(sa.seg_attn_bwd(Q, K, V, O, lse, dO, 256, 64, [0, 1]))
    sa.poll_status()
    sa.rope_rotate(X, table, positions=bad)
    O, lse = sa.seg_attn_fwd(Q, K, V, 256, 64, [0, 1])
    got = (O, lse) + tuple(sa.seg_attn_bwd(Q, K, V, O, lse, dO, 256, 64, [0, 1]))
    with pytest.raises(sa.SegAttnError) as e:
        sa.poll_status()
    assert e.value.status == 1
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_agrees_with_the_half_rotation_of_the_framework():
    X = torch.randn(2, 100, 4, 128, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    table = sa.rope_table(200, 128)
    a, b = sa.rope_apply(X, table, pos0=50).float(), sa.rope_rotate(X, table, pos0=50).float()
    # the older kernel contracts a product and a sum: before the rounding they differ by two fp32 roundings at most
    assert ((a - b).abs() <= 2 * ref.BF16 * b.abs() + 1e-6).all()
