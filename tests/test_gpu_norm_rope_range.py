"""Norms of rows whose squares leave fp32, with eps = 0 or far below them: as precise as others', in both directions and on the way into pages
(bounds: tests/e4m3.py and tests/test_gpu_norm_rope.py)."""
import numpy as np
import pytest
import torch

import oracle.e4m3 as orc
import paper_2604_10103_amd as hf
from e4m3 import UNIT, Batch8, norm_bound, pair_sizes, rope_of
from paged import DEV, HALF, TYPES, f64

from test_gpu_append_e4m3 import _append

pytestmark = pytest.mark.gpu

SIZES = [-140, -125, -90, -76, -70, -62, -51, -49, 0, 49, 51, 58, 61, 66, 90, 120]   # rows of about 2^this
TURNS = {"alone": {}, "adjacent": dict(pairs=[11, 9], halves=False), "halves": dict(pairs=[16, 8]), "odd": dict(pairs=[5, 4])}


def _rows(dtype, d, seed):
    """[1, 3, SIZES, d]"""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(1, 3, len(SIZES), d, generator=g, dtype=torch.float64) * torch.exp2(torch.tensor(SIZES, dtype=torch.float64))[:, None]
    if dtype == "bf16":
        x[..., SIZES.index(-140), :] *= 2.0 ** 10             # (bf16 ends at 2^-133)
    return x.to(TYPES[dtype]).to(DEV), g


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("turn", list(TURNS))
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30])
def test_rows_of_all_sizes(dtype, d, turn, eps):
    x, g = _rows(dtype, d, d)
    how = TURNS[turn]
    w = torch.randn(3, d, generator=g).to(DEV)
    pos = torch.randint(0, 900, (len(how["pairs"]), len(SIZES)), generator=g, dtype=torch.int32).to(DEV) if how else None
    own = dict(norm=hf.make_head_norm(eps, True), weight=w, positions=pos)
    if how:
        own["rope"] = rope_of(how["pairs"], how.get("halves", True))
    ref = dict(weight=f64(w), eps=float(np.float32(eps)), positions=None if pos is None else pos.cpu().numpy(), **how)
    y = torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, **own)
    want = orc.norm_turn(f64(x[0]), **ref)
    far = np.abs(f64(y[0]) - want) - norm_bound(f64(x[0]), dtype, want, **ref)
    assert (far <= 0).all(), [(s, float(v)) for s, v in zip(SIZES, far.max((0, 2))) if not v <= 0]
    # gradients, of a size that leaves dX in the type's range
    dy = torch.randn(1, 3, len(SIZES), d, generator=g) * torch.exp2(torch.tensor([40.0 if s > 0 else -40.0 if s < 0 else 0.0 for s in SIZES]))[:, None]
    dy = dy.to(x.dtype).to(DEV)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(own["norm"], d, 1, 3, len(SIZES)), dtype=torch.uint8, device=DEV)
    hf.hf_norm_rope_bwd(x, dy, dx, dweight=dw, workspace=ws, **own)
    want, rows_w = orc.norm_turn_gradient(f64(x[0]), f64(dy[0]), **ref)
    u, r = orc.norm(f64(x[0]), ref["eps"])
    G = pair_sizes(np.abs(f64(dy[0])), how.get("pairs"), how.get("halves", True), 1.0)
    wG = G * np.abs(f64(w))[:, None]
    bound = HALF[dtype] * np.abs(want) + UNIT * r * (32 * wG + 96 * np.abs(u) * (wG * np.abs(u)).mean(-1, keepdims=True))
    far = np.abs(f64(dx[0]) - want) - bound
    assert (far <= 0).all(), [(s, float(v)) for s, v in zip(SIZES, far.max((0, 2))) if not v <= 0]
    assert (np.abs(f64(dw) - rows_w.sum(1)) <= UNIT * (36 + len(SIZES) + 160) * (G * np.abs(u)).sum(1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by", [-100, 72])
def test_a_power_of_two_changes_nothing(dtype, by):
    """Without eps a row and its product with a power of two have the same norm: to the bit, where the kernel takes the same squares."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(1, 4, 50, 128, generator=g).to(TYPES[dtype]).to(DEV)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)[None]
    how = dict(norm=hf.make_head_norm(0.0), weight=torch.randn(128, generator=g).to(DEV), rope=rope_of([32]), positions=pos)
    y, z = torch.empty_like(x), torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, **how)
    hf.hf_norm_rope_fwd(x * 2.0 ** by, z, **how)
    assert torch.equal(y, z)
    new, lens = [30, 1], [50, 9]
    got = []
    for k in (0, by):
        b = Batch8(new, lens, 4, 2, 128, dtype, 16, seed=6)
        b.Q.mul_(2.0 ** k)
        b.K.mul_(2.0 ** k)
        out = _append(b, norm=how["norm"], k_weight=how["weight"], q_weight=how["weight"], rope=how["rope"])
        got.append((out, b.K_pages.view(torch.uint8), b.K_scales, b.V_pages.view(torch.uint8)))
    assert all(torch.equal(p, q) for p, q in zip(*got))


def test_the_largest_rows():
    """Without a rotation 15 of the bound's 21 units are counted."""
    top = torch.finfo(torch.float32).max
    x = torch.tensor([1.0, -1.0, 0.5, 2.0 ** -60]).repeat(16).mul(top)[None, None].to(DEV)
    y = torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, norm=hf.make_head_norm(0.0))
    want = orc.norm(f64(x), 0.0)[0]
    assert (np.abs(f64(y) - want) <= 21 * UNIT * np.abs(want)).all()


def test_rows_below_a_large_eps():
    """An eps beyond 2^100 leaves small rows small: no bit is lost until the results are subnormal."""
    x, _ = _rows("f32", 64, 3)
    y = torch.empty_like(x)
    for eps in (1e29, 1e33, 3e38):
        hf.hf_norm_rope_fwd(x, y, norm=hf.make_head_norm(eps))
        want = orc.norm(f64(x), float(np.float32(eps)))[0]
        assert (np.abs(f64(y) - want) <= 21 * UNIT * np.abs(want) + 2.0 ** -149).all()


def test_what_has_no_norm_has_none():
    x = torch.full((1, 1, 4, 64), 2.0 ** -80, device=DEV)
    x[0, 0, 1, 3], x[0, 0, 2, 3] = float("nan"), float("inf")
    x[0, 0, 3] = 0.0
    y = torch.empty_like(x)
    hf.hf_norm_rope_fwd(x, y, norm=hf.make_head_norm(0.0))
    assert (y[0, 0, 0] == 1).all() and torch.isnan(y[0, 0, 1]).all() and torch.isnan(y[0, 0, 3]).all()
    assert torch.isnan(y[0, 0, 2, 3]) and (y[0, 0, 2, :3] == 0).all()
    hf.hf_norm_rope_fwd(x, y, norm=hf.make_head_norm(1e-38))
    assert (y[0, 0, 3] == 0).all()
