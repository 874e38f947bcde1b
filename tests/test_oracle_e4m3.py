"""Pins of the 64-bit oracle of norms with rotation and of the pages in 8 bits."""
import math

import numpy as np
import pytest
import torch

import oracle.e4m3 as orc
import oracle.paged as paged


def test_codes_are_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(orc.e4m3_values(), got)


def test_quantised_rows_are_torchs_conversion():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(500, 64, generator=g) * (2 * torch.randn(500, 1, generator=g)).exp()
    x[0], x[1, 5], x[2, 7], x[3] = 0.0, math.nan, -math.inf, x[3] * 2.0 ** -130   # (x[3]: the smallest scale there is)
    scale = (x.abs().amax(-1) * (1.0 / 448.0)).clamp_min(2.0 ** -126)
    want = (x / scale[:, None]).to(torch.float8_e4m3fn).double().numpy()
    value, got = orc.quantise(x.double().numpy())
    fine = [i for i in range(500) if i not in (1, 2)]
    np.testing.assert_allclose(got[fine], scale.double().numpy()[fine], rtol=2.0 ** -23)
    assert (value[fine] == want[fine]).mean() > 0.999                            # (the scale's own rounding moves ties)
    assert np.isnan(got[1:3]).all() and (value[1:3] == 0).all() and (value[0] == 0).all()


@pytest.mark.parametrize("per_head", [False, True])
def test_norm_and_its_gradient_are_autograds(per_head):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(2, 3, 7, 16, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(*((3, 16) if per_head else (16,)), generator=g, dtype=torch.float64, requires_grad=True)
    pos = torch.randint(0, 50, (2, 7), generator=g).numpy()
    how = dict(pairs=[3, 2], halves=False, factor=4.0, trained=40.0, slow=0.1, fast=3.0, axes=(0, 1), amplitude=1.2)
    u = torch.nn.functional.rms_norm(x, (16,), eps=1e-3)
    y = u * (w[:, None] if per_head else w)
    rate = orc.rates([3, 2], factor=4.0, trained=40.0, slow=0.1, fast=3.0, axes=(0, 1))
    angle = torch.stack([torch.tensor(pos[a]).double() * r for a, r in rate], -1)
    z = torch.view_as_complex(y[..., :10].reshape(*y.shape[:-1], 5, 2)) * torch.polar(torch.full_like(angle, 1.2), angle)
    y = torch.cat([torch.view_as_real(z).flatten(-2), y[..., 10:]], -1)
    np.testing.assert_allclose(orc.norm_turn(x.detach().numpy(), w.detach().numpy(), 1e-3, pos, **how), y.detach().numpy(), atol=1e-12)
    dy = torch.randn(y.shape, generator=g, dtype=torch.float64)
    y.backward(dy)
    dX, dW = orc.norm_turn_gradient(x.detach().numpy(), dy.numpy(), w.detach().numpy(), 1e-3, pos, **how)
    np.testing.assert_allclose(dX, x.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(dW.sum((0, 2)) if per_head else dW.sum((0, 1, 2)), w.grad.numpy(), atol=1e-11)


def test_scaled_rates():
    plain = orc.rates([8, 8], shared=False)
    scaled = orc.rates([8, 8], shared=False, factor=8.0, trained=1000.0, slow=1.0, fast=32.0, axes=(1,))
    assert scaled[:8] == plain[:8] and scaled[8] == plain[8]                     # the other axis; 159 turns
    for (_, w), (_, s) in zip(plain[8:], scaled[8:]):
        turns = 1000.0 * w / (2 * math.pi)
        assert s == pytest.approx(w / 8 if turns <= 1 else w if turns >= 32 else w * ((turns - 1) / 31 * 7 / 8 + 1 / 8), rel=1e-12)
    np.testing.assert_array_equal(orc.turn(np.ones((3, 4, 32)), np.arange(8).reshape(2, 4), [8, 8]),
                                  paged.rotate_axes(np.ones((3, 4, 32)), np.arange(8).reshape(2, 4), [8, 8]))
