"""Small rows enter the pages in 8 bits as large ones do: to the bit, next to ties between codes and with a scale down to the least."""
import pytest
import torch

from e4m3 import Batch8

from test_gpu_append_e4m3 import _append

pytestmark = pytest.mark.gpu

TOP = list(range(-118, -80, 2))                               # rows' largest values, powers of two


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["f32", "bf16"])
def test_small_rows_are_quantised_to_the_bit(d, form):
    """A feature is one of the middles between two codes times the scale, rounded to the type, or up to two steps beside it."""
    n = 40 * len(TOP)
    b = Batch8([n], [n], 2, 1, d, form, 32, seed=d)
    g = torch.Generator().manual_seed(d)
    top = torch.exp2(torch.tensor(TOP).repeat(40)[:, None, None].float()) * (1 + torch.rand(n, 4, 1, generator=g))
    top = top.to(b.t).float()
    scale = torch.clamp(top * (1.0 / 448.0), min=2.0 ** -126)
    normal = (2 * torch.randint(8, 16, (n, 4, d), generator=g) + 1) / 16 * torch.exp2(torch.randint(-6, 8, (n, 4, d), generator=g).float())
    small = (2 * torch.randint(0, 8, (n, 4, d), generator=g) + 1) * 2.0 ** -10   # (codes below 2^-6 are 2^-9 apart)
    x = torch.where(torch.rand(n, 4, d, generator=g) < 0.3, small, normal) * scale
    if form == "f32":
        x = (x.view(torch.int32) + torch.randint(-2, 3, (n, 4, d), generator=g, dtype=torch.int32)).view(torch.float32)
    x = x.clamp_max(top) * torch.where(torch.rand(n, 4, d, generator=g) < 0.5, -1.0, 1.0)
    x[..., 5] = top[..., 0]
    b.rows.copy_(x.to(b.t))
    _append(b)
    page, place = torch.tensor(b.table[0])[torch.arange(n) // 32].long(), torch.arange(n) % 32
    for rows, codes, scales in ((b.K, b.K_pages, b.K_scales), (b.V, b.V_pages, b.V_scales)):
        y = rows.float().cpu()
        scale = torch.clamp(y.abs().amax(-1) * (1.0 / 448.0), min=2.0 ** -126)
        assert torch.equal(scales.cpu()[page, :, place], scale)
        want = (y / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(codes.view(torch.uint8).cpu()[page, :, place], want)
