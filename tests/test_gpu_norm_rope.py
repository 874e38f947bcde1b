"""Norms of queries and keys with the rotation in the same pass, and their gradients, against the 64-bit oracle (bounds: tests/e4m3.py)."""
import numpy as np
import pytest
import torch

import oracle.e4m3 as orc
import paper_2604_10103_amd as hf
from e4m3 import UNIT, norm_bound, pair_sizes, rope_of
from paged import DEV, HALF, TYPES, f64

pytestmark = pytest.mark.gpu

FORMS = {   # pairs of the axes by head_dim, layout, spectrum, scaling
    "alone": None,
    "adjacent": (lambda d: [d // 2 - 2 * (d // 6), d // 6, d // 6], False, False, None),
    "halves": (lambda d: [d // 4], True, True, None),
    "axes": (lambda d: [d // 8, d // 8], True, False, dict(factor=4.0, trained=300.0, slow=1.0, fast=20.0, amplitude=1.25, axes=(0,))),
    "odd": (lambda d: [5, 4], True, True, dict(factor=2.5, trained=50.0, slow=0.0, fast=2.0, amplitude=0.75, axes=(0, 1))),
    "few": (lambda d: [3], False, True, dict(factor=1.0, trained=50.0, amplitude=1.5, axes=())),
}


def _form(form, d):
    """The library's arguments, and the oracle's."""
    if FORMS[form] is None:
        return {}, {}
    pairs, halves, shared, scaling = FORMS[form]
    pairs = pairs(d)
    own = dict(rope=rope_of(pairs, halves, shared))
    ref = dict(pairs=pairs, halves=halves, shared=shared)
    if scaling:
        own["scaling"] = hf.make_rope_scaling(**scaling)
        ref.update(scaling)
    return own, ref


def _inputs(B, H, n, d, dtype, seed, weights, axes, per_batch=False, packed=False):
    g = torch.Generator().manual_seed(seed)
    shape = (B, n, H + 2, d) if packed else (B, H, n, d)
    x = torch.randn(shape, generator=g) * torch.randn(shape[:-1] + (1,), generator=g).exp()
    x = x.to(TYPES[dtype]).to(DEV)
    if packed:
        x = x[:, :, 1:H + 1].transpose(1, 2)
    w = {"none": None, "one": torch.randn(d, generator=g), "each": torch.randn(H, d, generator=g)}[weights]
    pos = torch.randint(-50, 5000, (B, axes, n) if per_batch else (axes, n), generator=g, dtype=torch.int32).to(DEV) if axes else None
    dy = torch.randn(B, H, n, d, generator=g).to(TYPES[dtype]).to(DEV)
    return x, None if w is None else w.to(DEV), pos, dy


def _by_batch(pos, b):
    return None if pos is None else (pos[b] if pos.dim() == 3 else pos).cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("weights", ["none", "one", "each"])
@pytest.mark.parametrize("B,H,n", [(1, 1, 1), (2, 7, 33), (3, 5, 130)])
def test_forward(dtype, d, form, weights, B, H, n):
    own, ref = _form(form, d)
    x, w, pos, _ = _inputs(B, H, n, d, dtype, n + d, weights, len(ref.get("pairs", [])), per_batch=B == 3, packed=H == 5)
    eps = 1e-5
    y = torch.full((B, H, n, d), 7.0, dtype=x.dtype, device=DEV)
    hf.hf_norm_rope_fwd(x, y, norm=hf.make_head_norm(eps, weights == "each"), weight=w, positions=pos, **own)
    for b in range(B):
        how = dict(weight=None if w is None else f64(w), eps=float(np.float32(eps)), positions=_by_batch(pos, b), **ref)
        want = orc.norm_turn(f64(x[b]), **how)
        far = np.abs(f64(y[b]) - want) - norm_bound(f64(x[b]), dtype, want, **how)
        assert (far <= 0).all(), far.max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", [f for f in FORMS if f != "alone"])
def test_without_norm_it_is_the_rotation(dtype, form):
    """(Which product of a pair's sum is rounded before it is the compiler's choice: equal bits are not promised.)"""
    own, ref = _form(form, 64)
    x, _, pos, dy = _inputs(2, 3, 40, 64, dtype, 3, "none", len(ref["pairs"]))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, positions=pos, **own)
    hf.hf_norm_rope_bwd(x, dy, dx, positions=pos, **own)
    how = dict(positions=_by_batch(pos, 0), **ref)
    for got, rows, back in ((y, x, False), (dx, dy, True)):
        for b in range(2):
            r = orc.turn(f64(rows[b]), inverse=back, **how)
            assert (np.abs(f64(got[b]) - r) <= norm_bound(f64(rows[b]), dtype, r, **how)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_packed_and_strided(dtype):
    g = torch.Generator().manual_seed(11)
    rows = torch.randn(37, 9, 128, generator=g).to(TYPES[dtype]).to(DEV)
    rope, norm = rope_of([40]), hf.make_head_norm()
    w = torch.randn(128, generator=g).to(DEV)
    pos = torch.arange(37, dtype=torch.int32, device=DEV)[None]
    y = torch.empty(37, 4, 128, dtype=rows.dtype, device=DEV)
    before = rows.clone()
    hf.hf_norm_rope_fwd(rows[:, 2:6], y, norm=norm, weight=w, rope=rope, positions=pos)
    hf.hf_norm_rope_fwd(rows[:, 2:6], rows[:, 2:6], norm=norm, weight=w, rope=rope, positions=pos)
    assert torch.equal(rows[:, 2:6], y) and torch.equal(rows[:, :2], before[:, :2]) and torch.equal(rows[:, 6:], before[:, 6:])
    # a head's rows shared by all heads: stride zero
    z = torch.empty(2, 5, 37, 128, dtype=rows.dtype, device=DEV)
    x = before[:, 0].expand(2, 5, 37, 128)
    hf.hf_norm_rope_fwd(x, z, norm=norm, weight=w, rope=rope, positions=pos)
    one = torch.empty(37, 1, 128, dtype=rows.dtype, device=DEV)
    hf.hf_norm_rope_fwd(before[:, :1].contiguous(), one, norm=norm, weight=w, rope=rope, positions=pos)
    assert all(torch.equal(z[b, h], one[:, 0]) for b in range(2) for h in range(5))
    # gradients into X and into dY
    dy = torch.randn(37, 4, 128, generator=g).to(rows.dtype).to(DEV)
    dx = torch.empty_like(dy)
    x4 = before[:, 2:6].contiguous()
    hf.hf_norm_rope_bwd(x4, dy, dx, norm=norm, weight=w, rope=rope, positions=pos)
    for into in (0, 1):
        a, b = x4.clone(), dy.clone()
        hf.hf_norm_rope_bwd(a, b, (a, b)[into], norm=norm, weight=w, rope=rope, positions=pos)
        assert torch.equal((a, b)[into], dx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("weights", ["none", "one", "each"])
@pytest.mark.parametrize("B,H,n", [(1, 1, 1), (2, 7, 33), (3, 5, 130)])
def test_gradients(dtype, d, form, weights, B, H, n):
    """With G the sizes that turn back to g (21 units off, as in the forward pass), u 13 units: a product of both is 36 units off, its mean
    over the row 36 + 24 more for the sum; dX's two terms and their difference, times r (13): within 32 units of r |w G| and 96 of
    r |u| mean |w G u|; then a rounding to the type.  dweight sums B H n such products in some order: at most as many roundings and 160."""
    own, ref = _form(form, d)
    x, w, pos, dy = _inputs(B, H, n, d, dtype, n + d, weights, len(ref.get("pairs", [])), per_batch=B == 3, packed=H == 5)
    eps = 1e-5
    norm = hf.make_head_norm(eps, weights == "each")
    dx = torch.full((B, H, n, d), 7.0, dtype=x.dtype, device=DEV)
    dw = torch.full((H, d) if weights == "each" else (d,), 7.0, device=DEV)
    ws = torch.randint(0, 255, (hf.hf_norm_rope_bwd_workspace_bytes(norm, d, B, H, n),), dtype=torch.uint8, device=DEV)
    hf.hf_norm_rope_bwd(x, dy, dx, norm=norm, weight=w, positions=pos, dweight=dw, workspace=ws, **own)
    want_w, bound_w = 0.0, 0.0
    for b in range(B):
        w64 = None if w is None else f64(w)
        want, rows_w = orc.norm_turn_gradient(f64(x[b]), f64(dy[b]), weight=w64, eps=float(np.float32(eps)), positions=_by_batch(pos, b), **ref)
        u, r = orc.norm(f64(x[b]), float(np.float32(eps)))
        G = pair_sizes(np.abs(f64(dy[b])), ref.get("pairs"), ref.get("halves", True), ref.get("amplitude", 1.0))
        wG = G if w64 is None else G * np.abs(w64[:, None] if w64.ndim == 2 else w64)
        bound = HALF[dtype] * np.abs(want) + UNIT * r * (32 * wG + 96 * np.abs(u) * (wG * np.abs(u)).mean(-1, keepdims=True))
        far = np.abs(f64(dx[b]) - want) - bound
        assert (far <= 0).all(), far.max()
        want_w = want_w + rows_w.sum(1)
        bound_w = bound_w + (G * np.abs(u)).sum(1)
    if weights != "each":
        want_w, bound_w = want_w.sum(0), bound_w.sum(0)
    assert (np.abs(f64(dw) - want_w) <= UNIT * (36 + B * H * n + 160) * bound_w).all()
    again = torch.empty_like(dw)
    hf.hf_norm_rope_bwd(x, dy, dx, norm=norm, weight=w, positions=pos, dweight=again, workspace=ws, **own)
    assert torch.equal(again, dw)


def test_gradients_are_differences():
    """Central differences of the forward call in fp32, step h: off by the forward's rounding over h, and by h^2 of the third derivative."""
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(1, 2, 3, 64, generator=g).to(DEV), torch.randn(2, 64, generator=g).to(DEV)
    dy = torch.randn(1, 2, 3, 64, generator=g).to(DEV)
    pos = torch.arange(3, dtype=torch.int32, device=DEV)[None]
    how = dict(norm=hf.make_head_norm(1e-3, True), rope=rope_of([24]), positions=pos, scaling=hf.make_rope_scaling(2.0, 20.0, 0.1, 1.0, 1.1))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(how["norm"], 64, 1, 2, 3), dtype=torch.uint8, device=DEV)
    hf.hf_norm_rope_bwd(x, dy, dx, weight=w, dweight=dw, workspace=ws, **how)

    def loss(x, w):
        y = torch.empty_like(x)
        hf.hf_norm_rope_fwd(x, y, weight=w, **how)
        return float((y.double() * dy.double()).sum())

    h = 2.0 ** -6
    for t, grad in ((x, dx), (w, dw)):
        for at in range(0, t.numel(), 37):
            up, down = t.clone(), t.clone()
            up.view(-1)[at] += h
            down.view(-1)[at] -= h
            d = (loss(up, w) - loss(down, w)) / (2 * h) if t is x else (loss(x, up) - loss(x, down)) / (2 * h)
            # a loss of up to 128 products of size 10 at 21 units each: 1.6e-3 h^-1 2^-10; third derivatives of size 30 here
            assert abs(d - float(grad.view(-1)[at])) <= 128 * 10 * 21 * UNIT / h + 30 * h * h


@pytest.mark.parametrize("per_head", [False, True])
def test_many_tokens_and_heads(per_head):
    """Workgroups that stay for several tokens; more heads and batches than there are workgroups for."""
    for B, H, n, d in ((2, 12, 3001, 128), (70, 20, 3, 64), (1, 1, 20001, 64)):
        x, w, pos, dy = _inputs(B, H, n, d, "f32", 5, "each" if per_head else "one", 1)
        norm = hf.make_head_norm(1e-6, per_head)
        rope = rope_of([16])
        dx, dw = torch.empty(B, H, n, d, device=DEV), torch.empty_like(w)
        ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(norm, d, B, H, n), dtype=torch.uint8, device=DEV)
        hf.hf_norm_rope_bwd(x, dy, dx, norm=norm, weight=w, rope=rope, positions=pos, dweight=dw, workspace=ws)
        want, rows_w = orc.norm_turn_gradient(f64(x), f64(dy), f64(w), float(np.float32(1e-6)), _by_batch(pos, 0), pairs=[16])
        u, r = orc.norm(f64(x), float(np.float32(1e-6)))
        G = pair_sizes(np.abs(f64(dy)), [16], True, 1.0)
        wG = G * np.abs(f64(w)[:, None] if per_head else f64(w))
        bound = UNIT * np.abs(want) + UNIT * r * (32 * wG + 96 * np.abs(u) * (wG * np.abs(u)).mean(-1, keepdims=True))
        assert (np.abs(f64(dx) - want) <= bound).all()
        axes = (0, 2) if per_head else (0, 1, 2)
        # (in fact a chain of some hundred additions, then a tree of the rest)
        assert (np.abs(f64(dw) - rows_w.sum(axes)) <= UNIT * (36 + 1500) * (G * np.abs(u)).sum(axes)).all()


def test_no_tokens_and_values_that_are_not_finite():
    norm = hf.make_head_norm(0.0)
    empty = torch.empty(2, 3, 0, 64, device=DEV)
    dw = torch.full((64,), 7.0, device=DEV)
    hf.hf_norm_rope_fwd(empty, empty, norm=norm)
    hf.hf_norm_rope_bwd(empty, empty, empty, norm=norm, dweight=dw)
    assert (dw == 0).all()
    x = torch.ones(1, 1, 5, 64, device=DEV)
    x[0, 0, 1, 3], x[0, 0, 2, 3] = float("nan"), float("inf")
    x[0, 0, 3] = 0.0
    y = torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, norm=norm)
    assert (y[0, 0, [0, 4]] == 1).all() and torch.isnan(y[0, 0, 1]).all() and torch.isnan(y[0, 0, 3]).all()
    assert torch.isnan(y[0, 0, 2, 3]) and (y[0, 0, 2, :3] == 0).all()


def test_streams_and_graphs():
    x, w, pos, dy = _inputs(2, 6, 300, 128, "bf16", 9, "one", 1)
    norm, rope = hf.make_head_norm(), rope_of([64])
    y, dx, dw = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(w)
    ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(norm, 128, 2, 6, 300), dtype=torch.uint8, device=DEV)

    def step(y, dx, dw, ws):
        hf.hf_norm_rope_fwd(x, y, norm=norm, weight=w, rope=rope, positions=pos)
        hf.hf_norm_rope_bwd(x, dy, dx, norm=norm, weight=w, rope=rope, positions=pos, dweight=dw, workspace=ws)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(y, dx, dw, ws)
    for k in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(k)).to(x.dtype))
        graph.replay()
        torch.cuda.synchronize()
        y2, dx2, dw2 = torch.empty_like(y), torch.empty_like(dx), torch.empty_like(dw)
        step(y2, dx2, dw2, torch.empty_like(ws))
        assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
