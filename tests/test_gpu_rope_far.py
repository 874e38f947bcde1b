"""Sines and cosines of the rotation by positions as the header bounds them: off by 2.5 units of 2^-24 at most, whatever the position.

Rows of (1, 0) pairs turn into (cos, sin) as they are.  The reference's angles have 60 digits: in 64 bits a rate's rounding alone moves the
angle of a position of 2^31 by more than the bound."""
import math
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2604_10103_amd as hf
from paged import DEV, Batch

pytestmark = pytest.mark.gpu

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
FAR = [0, 1, -1, 77, 4096, 100001, 1 << 20, -(1 << 24) + 1, (1 << 28) - 57, (1 << 30) + 12345, 2000000011, -1999999973, (1 << 31) - 1, (1 << 31) - 2,
       -(1 << 31), -(1 << 31) + 1, 1717986918, -1431655765]


def _cos_sin(pos, pairs, theta, shared):
    """[axes, n] positions -> cosines and sines [n, P]; the angle is reduced to [-pi/4, pi/4] in 60 digits."""
    P, out, p = sum(pairs), [], 0
    for a, count in enumerate(pairs):
        for i in range(count):
            power = Decimal(p) / P if shared else Decimal(i) / count
            rate = (-power * Decimal(theta).ln()).exp()
            for x in pos[a]:
                angle = Decimal(int(x)) * rate
                turns = (angle * 2 / PI).to_integral_value()
                r = float(angle - turns * PI / 2)
                c, s = math.cos(r), math.sin(r)
                out.append([(c, s), (-s, c), (-c, -s), (s, -c)][int(turns) % 4])
            p += 1
    return np.array(out).reshape(P, len(pos[0]), 2).transpose(1, 0, 2)


@pytest.mark.parametrize("pairs,halves,shared,theta,d", [([32], True, True, 10000.0, 64), ([22, 21, 21], False, False, 10000.0, 128),
                                                         ([16, 24, 24], True, True, 1e6, 128), ([9, 4], True, False, 500000.0, 64),
                                                         ([1, 3], False, True, 1.0, 64)])
@pytest.mark.parametrize("inverse", [False, True])
def test_any_position(pairs, halves, shared, theta, d, inverse):
    P, n = sum(pairs), len(FAR)
    pos = np.array([np.roll(FAR, 5 * a) for a in range(len(pairs))], dtype=np.int64)
    X = torch.zeros((1, 1, n, d))
    re = np.arange(P) if halves else 2 * np.arange(P)
    im = re + P if halves else re + 1
    X[..., re] = 1.0
    Y = torch.empty((1, 1, n, d), device=DEV)
    rope = hf.make_rope_axes(pairs, theta=theta, layout=hf.HF_ROPE_HALVES if halves else hf.HF_ROPE_ADJACENT,
                             spectrum=hf.HF_ROPE_SHARED if shared else hf.HF_ROPE_PER_AXIS)
    hf.hf_rope_axes_apply(rope, X.to(DEV), torch.tensor(pos, dtype=torch.int32, device=DEV), Y, inverse=inverse)
    got, ref = Y[0, 0].double().cpu().numpy(), _cos_sin(pos, pairs, theta, shared)
    off = np.maximum(np.abs(got[:, re] - ref[..., 0]), np.abs(got[:, im] - (-1 if inverse else 1) * ref[..., 1])).max(1) * 2.0 ** 24
    assert (off <= 2.5).all(), dict(zip(pos[0].tolist(), off.tolist()))


def test_keys_far_behind():
    """The append turns keys by the same angles."""
    b = Batch([len(FAR)], [len(FAR)], 2, 1, 64, "f32", 32)
    b.rows.zero_()
    b.rows[..., :32] = 1.0
    pos = np.array([FAR], dtype=np.int64)
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d, rope=hf.make_rope_axes([32]),
                       positions=torch.tensor(pos, dtype=torch.int32, device=DEV))
    got, ref = b.K_pages[int(b.table[0, 0]), 0, :len(FAR)].double().cpu().numpy(), _cos_sin(pos, [32], 10000.0, True)
    assert np.abs(got - np.concatenate([ref[..., 0], ref[..., 1]], -1)).max() <= 2.5 * 2.0 ** -24
