"""The gradient of the norms' weights over many rows: as precise as over few.  More batches or heads than there are workgroups leave a thread
hundreds of rows; they are read from a few by strides of zero, so that the 64-bit answer is a small one's multiple."""
import numpy as np
import pytest
import torch

import oracle.e4m3 as orc
import paper_2604_10103_amd as hf
from e4m3 import UNIT
from paged import DEV, f64

pytestmark = pytest.mark.gpu

MANY, EPS = 1024, 1e-6


def _gradient(x, dy, w, per_head):
    """dweight of x, dy [1, 1, tokens, d], read MANY times: as batches, or as heads with weights of their own."""
    n, d = x.shape[2], x.shape[3]
    shape = (1, MANY, n, d) if per_head else (MANY, 1, n, d)
    norm = hf.make_head_norm(EPS, per_head)
    weight = w.expand(MANY, d).contiguous() if per_head else w
    dx, dw = torch.empty(shape, device=DEV), torch.empty_like(weight)
    ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(norm, d, shape[0], shape[1], n), dtype=torch.uint8, device=DEV)
    hf.hf_norm_rope_bwd(x.expand(shape), dy.expand(shape), dx, norm=norm, weight=weight, dweight=dw, workspace=ws)
    again = torch.empty_like(dw)
    hf.hf_norm_rope_bwd(x.expand(shape), dy.expand(shape), dx, norm=norm, weight=weight, dweight=again, workspace=ws)
    assert torch.equal(dw, again)
    return f64(dw)


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("d,n", [(128, 16 * 600), (64, 32 * 600), (128, 16 * 17 + 5)])
@pytest.mark.parametrize("rows", ["equal", "any"])
def test_many_rows_of_a_thread(per_head, d, n, rows):
    """Without a rotation a product of dY and u is 15 units off (u: r's 13, its product; its own rounding).  16 rows are summed in fp32, 16
    roundings at most, those sums in 64 bits; a workgroup's is rounded once, and so is the gradient: 33 units of the products' sizes, however
    many there are.  (Equal rows err the same way every time.)"""
    g = torch.Generator().manual_seed(d + n)
    shape = (1, 1, n if rows == "any" else 1, d)
    x, dy, w = torch.randn(shape, generator=g).to(DEV), torch.randn(shape, generator=g).to(DEV), torch.randn(d, generator=g).to(DEV)
    u, _ = orc.norm(f64(x), float(np.float32(EPS)))
    t = (f64(dy) * u)[0, 0]
    times = (n if rows == "equal" else 1) * (1 if per_head else MANY)
    if rows == "equal":
        x, dy = x.expand(1, 1, n, d), dy.expand(1, 1, n, d)
    got = _gradient(x, dy, w, per_head)
    far = np.abs(got - times * t.sum(0)) / (times * np.abs(t).sum(0))
    assert (far <= 33 * UNIT).all(), far.max() / UNIT
