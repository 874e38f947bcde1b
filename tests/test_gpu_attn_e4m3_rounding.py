"""Attention over pages in 8 bits: what calls of few rows round, element by element against the 64-bit oracle."""
import numpy as np
import pytest

from e4m3 import UNIT, Batch8
from paged import HALF, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,lens,heads,heads_kv", [
    ([1], [700], 8, 2), ([1] * 4, [90, 2100, 33, 1000], 8, 8), ([4], [3000], 16, 4), ([7, 1], [900, 400], 8, 2), ([1], [1500], 32, 1),
    # four wavefronts a row tile, and one
    ([1] * 60, [20 + 7 * i for i in range(60)], 8, 8), ([1] * 300, [20 + i % 70 for i in range(300)], 8, 8)])
def test_few_rows_round_bf16_outputs_once(d, new, lens, heads, heads_kv):
    """Products of probability and scale go to the second product as two bf16, the second the rounding of what the first left: 2^-16 of
    their size is lost.  The rest is the bound of fp32 pages (scores: 3 d + 8 more roundings than products, sums: n + 64), and one
    rounding of the output.  A single bf16 would leave 2^-8 of the probabilities' size, which most outputs near zero show."""
    b = Batch8(new, lens, heads, heads_kv, d, "bf16", 16, seed=d + len(lens))
    O, _ = b.attend(lse=False)
    R, _, spread, size, count = b.oracle()
    delta = (3 * d + 16) * UNIT * size[..., None]
    sums = (count[:, None, None] + 64) * UNIT
    bound = HALF["bf16"] * np.abs(R) + spread * (2.0 ** -16 + 2 * delta + 2 * sums)
    far = np.abs(f64(O) - R) - bound
    assert (far <= 0).all(), f"{(far > 0).mean():.3e} of the values beyond the bound, by {far.max():.3e}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 2], [60, 3]])
@pytest.mark.parametrize("size", [-100, 100])
def test_values_of_the_sizes_that_keep_their_precision(dtype, new, size):
    """Scales of values between 2^-100 and 2^100: parts of p v_scale below 2^-134 are lost, 2^-30 of a sum of such sizes and less than one of
    the 64 roundings that the bound counts beside a sum's own; a sum of products of up to 2^8, 448 and 2^100 is finite."""
    b = Batch8(new, [300, 70], 4, 2, 64, dtype, 16, seed=3)
    top = float(b.V_scales.max())
    b.V_scales.mul_(2.0 ** size / top).clamp_min_(2.0 ** -100)
    b.check(*b.attend())
