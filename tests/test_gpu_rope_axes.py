"""Rotation by positions with several axes against the 64-bit oracle, element by element.

Bound: sine and cosine are off by 2.5 units of 2^-24, the two products and their sum by one each, of |x_a| + |x_b|; then one rounding
to the storage type."""
import numpy as np
import pytest
import torch

import oracle.paged as orc
import paper_2604_10103_amd as hf
from paged import DEV, HALF, TYPES, f64

pytestmark = pytest.mark.gpu


def _bound(x, ref, pairs, halves, dtype):
    P, part = sum(pairs), np.zeros_like(ref)
    for p in range(P):
        u, v = (p, p + P) if halves else (2 * p, 2 * p + 1)
        part[..., u] = part[..., v] = np.abs(x[..., u]) + np.abs(x[..., v])
    return HALF[dtype] * np.abs(ref) + 5 * 2.0 ** -24 * part


def _rope(pairs, halves=True, shared=True, theta=10000.0):
    return hf.make_rope_axes(pairs, theta=theta, layout=hf.HF_ROPE_HALVES if halves else hf.HF_ROPE_ADJACENT,
                             spectrum=hf.HF_ROPE_SHARED if shared else hf.HF_ROPE_PER_AXIS)


SHAPES = [   # pairs, halves, shared, d
    ([64], True, True, 128), ([16, 24, 24], True, True, 128), ([22, 21, 21], False, False, 128), ([12, 10, 10], False, False, 64),
    ([32], True, True, 64), ([8, 8, 8], True, True, 64), ([7, 6, 6], True, False, 64), ([5, 4, 3, 1], True, True, 128),
    ([3], False, True, 64), ([1, 1], True, True, 64), ([40, 24], False, True, 128), ([61], True, False, 128), ([32, 32], True, False, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,halves,shared,d", SHAPES)
@pytest.mark.parametrize("batch,heads,n", [(1, 1, 1), (2, 5, 37), (1, 9, 130)])
def test_forward_and_inverse_follow_the_formula(dtype, pairs, halves, shared, d, batch, heads, n):
    g = torch.Generator().manual_seed(n + heads)
    X = torch.randn((batch, heads, n, d), generator=g).to(TYPES[dtype])
    pos = torch.randint(-50, 100000, (len(pairs), n), generator=g, dtype=torch.int32)
    pos[0, -1] = 0
    for inverse in (False, True):
        Y = torch.full((batch, heads, n, d), 7.0, dtype=TYPES[dtype], device=DEV)
        hf.hf_rope_axes_apply(_rope(pairs, halves, shared), X.to(DEV), pos.to(DEV), Y, inverse=inverse)
        ref = orc.rotate_axes(f64(X), pos.numpy(), pairs, halves=halves, shared=shared, inverse=inverse)
        assert (np.abs(f64(Y) - ref) <= _bound(f64(X), ref, pairs, halves, dtype)).all()
        assert torch.equal(Y[..., 2 * sum(pairs):].cpu(), X[..., 2 * sum(pairs):])   # the others stay as they are


@pytest.mark.parametrize("far", [1 << 20, 1 << 24, (1 << 31) - 1])
def test_far_positions_are_reduced_in_64_bits(far):
    """The product of a position and a rate is off by 2^-52 of itself in either computation (the rate's rounding and its own)."""
    pairs, d = [32], 64
    X = torch.randn((1, 2, 4, d), generator=torch.Generator().manual_seed(1))
    pos = torch.tensor([[far, -far, far - 1, far // 3]], dtype=torch.int32)
    Y = torch.empty_like(X, device=DEV)
    hf.hf_rope_axes_apply(_rope(pairs), X.to(DEV), pos.to(DEV), Y)
    ref = orc.rotate_axes(f64(X), pos.numpy(), pairs)
    part = np.abs(f64(X))[..., :32] + np.abs(f64(X))[..., 32:]
    slack = far * 4 * 2.0 ** -52 * np.concatenate([part, part], -1)
    assert (np.abs(f64(Y) - ref) <= _bound(f64(X), ref, pairs, True, "f32") + slack).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,halves", [([22, 21, 21], False), ([16, 24, 24], True), ([9, 4], True)])
def test_views_packed_rows_and_in_place_give_the_same_bits(dtype, pairs, halves):
    n, H, d = 77, 6, 128
    g = torch.Generator().manual_seed(3)
    rows = torch.randn((n, H + 5, d), generator=g).to(TYPES[dtype]).to(DEV)
    pos = torch.randint(0, 5000, (len(pairs), n), generator=g, dtype=torch.int32).to(DEV)
    rope = _rope(pairs, halves)
    plain = rows[:, 2:2 + H].transpose(0, 1).contiguous()[None]
    want = torch.empty_like(plain)
    hf.hf_rope_axes_apply(rope, plain, pos, want)
    packed = torch.empty((n, H, d), dtype=rows.dtype, device=DEV)
    hf.hf_rope_axes_apply(rope, rows[:, 2:2 + H], pos, packed)
    assert torch.equal(packed.transpose(0, 1), want[0])
    view = torch.empty((1, H, n, d), dtype=rows.dtype, device=DEV)
    hf.hf_rope_axes_apply(rope, rows[:, 2:2 + H].transpose(0, 1)[None], pos, view)
    assert torch.equal(view, want)
    before = rows.clone()
    hf.hf_rope_axes_apply(rope, rows[:, 2:2 + H], pos, rows[:, 2:2 + H])
    assert torch.equal(rows[:, 2:2 + H].transpose(0, 1), want[0])
    assert torch.equal(rows[:, :2], before[:, :2]) and torch.equal(rows[:, 2 + H:], before[:, 2 + H:])
    one = plain[:, :1].expand(1, H, n, d)   # one head read for all
    hf.hf_rope_axes_apply(rope, one, pos, view)
    assert all(torch.equal(view[0, h], want[0, 0]) for h in range(H))


def test_positions_of_every_batch():
    B, H, n, d, pairs = 3, 2, 21, 64, [12, 10, 10]
    g = torch.Generator().manual_seed(4)
    X = torch.randn((B, H, n, d), generator=g).to(DEV)
    pos = torch.randint(0, 300, (B, 3, n), generator=g, dtype=torch.int32).to(DEV)
    rope, Y, one = _rope(pairs, False, False), torch.empty_like(X), torch.empty((1, H, n, d), device=DEV)
    hf.hf_rope_axes_apply(rope, X, pos, Y)
    for b in range(B):
        hf.hf_rope_axes_apply(rope, X[b:b + 1], pos[b].contiguous(), one)
        assert torch.equal(Y[b:b + 1], one)


def test_a_grid_is_what_the_tables_give():
    """The convention of hf_rope_tables: adjacent pairs, a spectrum per axis; tables are rounded to fp32 (2^-24 each)."""
    frames, h, w, pairs, d = [3, 4, 9], 5, 7, (22, 21, 21), 128
    n = len(frames) * h * w
    cs, sn = (torch.empty((n, 64), device=DEV) for _ in range(2))
    hf.hf_rope_tables(frames, h, w, pairs, cs, sn)
    X = torch.randn((1, 3, n, d), generator=torch.Generator().manual_seed(5)).to(DEV)
    cfg = hf.make_config(1, 3, d, "f32", 64, 64)
    a, b = torch.empty_like(X), torch.empty_like(X)
    hf.hf_rope_apply(cfg, X, cs, sn, a)
    t = torch.arange(n)
    pos = torch.stack([torch.tensor(frames)[t // (h * w)], t // w % h, t % w]).to(torch.int32).to(DEV)
    hf.hf_rope_axes_apply(_rope(pairs, False, False), X, pos, b)
    part = X.abs()[..., 0::2] + X.abs()[..., 1::2]
    assert ((a - b).abs() <= 10 * 2.0 ** -24 * part.repeat_interleave(2, -1)).all()


def test_inverse_is_the_gradient():
    """<dY, R x> = <R^-1 dY, x>, and R^-1 R x = x; central differences of a linear map are exact but for rounding."""
    pairs, d, n = [6, 5, 5], 64, 33
    g = torch.Generator().manual_seed(6)
    X, dY = (torch.randn((1, 4, n, d), generator=g).to(DEV) for _ in range(2))
    pos = torch.randint(0, 900, (3, n), generator=g, dtype=torch.int32).to(DEV)
    rope, Y, dX, back = _rope(pairs), torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
    hf.hf_rope_axes_apply(rope, X, pos, Y)
    hf.hf_rope_axes_apply(rope, dY, pos, dX, inverse=True)
    hf.hf_rope_axes_apply(rope, Y, pos, back, inverse=True)
    size = float((dY.double().abs() * Y.double().abs()).sum() + (dX.double().abs() * X.double().abs()).sum())
    assert abs(float((dY.double() * Y.double()).sum() - (dX.double() * X.double()).sum())) <= 10 * 2.0 ** -24 * size
    part = X.abs()[..., :16] + X.abs()[..., 16:32]
    assert ((back - X).abs()[..., :32] <= 20 * 2.0 ** -24 * torch.cat([part, part], -1)).all()
    eps, bump = 2.0 ** -3, torch.zeros_like(X)
    for f in (0, 15, 16, 31, 40):
        bump.zero_()
        bump[0, 1, 7, f] = eps
        hi, lo = torch.empty_like(X), torch.empty_like(X)
        hf.hf_rope_axes_apply(rope, X + bump, pos, hi)
        hf.hf_rope_axes_apply(rope, X - bump, pos, lo)
        num = float(((hi.double() - lo.double()) * dY.double()).sum() / (2 * eps))
        # two outputs differ, each off by 10 units of 2^-24 of its pair, divided by eps
        assert abs(num - float(dX[0, 1, 7, f])) <= 20 * 2.0 ** -24 / eps * 2 * float(X[0, 1, 7].abs().max() * 2 * dY[0, 1, 7].abs().max()) + 1e-6


def test_infinities_stay_in_their_pair():
    pairs, d = [8, 4], 64
    X = torch.ones((1, 1, 3, d))
    X[0, 0, 1, 2], X[0, 0, 1, 50], X[0, 0, 2, 63] = float("inf"), float("nan"), float("-inf")
    pos = torch.tensor([[0, 5, 9], [2, 2, 2]], dtype=torch.int32)
    for halves in (True, False):
        Y = torch.empty_like(X, device=DEV)
        hf.hf_rope_axes_apply(_rope(pairs, halves), X.to(DEV), pos.to(DEV), Y)
        bad = ~torch.isfinite(Y[0, 0].cpu())
        pair = (2, 14) if halves else (2, 3)
        assert not bad[0].any() and set(torch.nonzero(bad[1]).flatten().tolist()) <= {*pair, 50} and bad[1, 50]
        assert torch.nonzero(bad[2]).flatten().tolist() == [63]


def test_a_captured_call_follows_its_positions():
    pairs, d, n = [16, 24, 24], 128, 65
    X = torch.randn((1, 4, n, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    pos = torch.zeros((3, n), dtype=torch.int32, device=DEV)
    rope, Y, want = _rope(pairs), torch.empty_like(X), torch.empty_like(X)
    hf.hf_rope_axes_apply(rope, X, pos, Y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hf.hf_rope_axes_apply(rope, X, pos, Y)
    for k in range(4):
        pos += 17 + k
        Y.zero_()
        hf.hf_rope_axes_apply(rope, X, pos, want)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_other_streams():
    X = torch.randn((1, 4, 300, 64), generator=torch.Generator().manual_seed(9)).to(DEV)
    pos = torch.arange(300, dtype=torch.int32, device=DEV)[None]
    rope, want, Y = _rope([32]), torch.empty_like(X), torch.empty_like(X)
    hf.hf_rope_axes_apply(rope, X, pos, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        hf.hf_rope_axes_apply(rope, X, pos, Y)
    s.synchronize()
    assert torch.equal(Y, want)


def test_no_tokens():
    X = torch.empty((1, 4, 0, 64), device=DEV)
    hf.hf_rope_axes_apply(_rope([32]), X, torch.empty((1, 0), dtype=torch.int32, device=DEV), X)
