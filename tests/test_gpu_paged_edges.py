"""Attention over pages where the older tests assert nothing: rows that see a key that is infinite, and equal bits, sharp rows and strides
in the workgroups of 128 and 256 rows (bounds: tests/paged.py)."""
import numpy as np
import pytest
import torch

from paged import HALF, Batch, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
@pytest.mark.parametrize("mask", [dict(), dict(causal=False, window=30, n_sink=3)])
@pytest.mark.parametrize("new,lens", [([70, 1], [90, 50]), ([1, 3], [200, 64]), ([1, 1], [9000, 33])])
@pytest.mark.parametrize("page", [24, 64])
def test_infinite_keys(dtype, d, bad, mask, new, lens, page):
    """One infinite feature makes a score of +inf, and its row NaN, or of -inf, and the key counts for nothing."""
    b = Batch(new, lens, 6, 2, d, dtype, page, seed=41, **mask)
    _, _, _, size, count = b.oracle()                          # (sizes of the scores that stay finite)
    for s in (0, 1):
        for j, f in ((lens[s] - 1, 0), (lens[s] // 2, d - 1), (1, 5)):
            b.K_pages[int(b.table[s, j // page]), :, j % page, f] = bad
    with np.errstate(invalid="ignore"):
        R, L, spread, _, _ = b.oracle()
    O, lse2 = b.attend()
    got, got_lse, lost = f64(O), f64(lse2), np.isnan(L.T)
    assert lost.any() and not lost.all()
    assert np.isnan(got[lost]).all() and np.isnan(got_lse.T[lost]).all()
    delta = ((d + 8) * 2.0 ** -24 * size)[..., None]
    sums = (count[:, None, None] + 64) * 2.0 ** -24
    bound = HALF[dtype] * np.abs(R) + spread * ((HALF["bf16"] if dtype == "bf16" else 0.0) + 2 * delta + 2 * sums)
    assert (np.abs(got - R) <= bound)[~lost].all()
    assert (np.abs(got_lse.T - L.T) <= 1.5 * (delta + 2 * sums)[..., 0] + 2.0 ** -22 * np.abs(L.T))[~lost].all()


LARGE = [   # new tokens, lengths, heads, key heads, d, type: workgroups of 128 rows but for the third and fourth, of 256
    ([300, 1, 70], [2000, 4000, 70], 8, 2, 128, "bf16"), ([300, 1, 70], [2000, 4000, 70], 8, 2, 64, "bf16"),
    ([1030, 5, 131], [1300, 400, 131], 32, 32, 128, "bf16"), ([700, 900], [1500, 900], 32, 16, 128, "bf16"),
    ([300, 1, 70], [2000, 4000, 70], 8, 2, 128, "f32"), ([300, 1, 70], [2000, 4000, 70], 8, 2, 64, "f32")]


@pytest.mark.parametrize("new,lens,heads,heads_kv,d,dtype", LARGE)
@pytest.mark.parametrize("page", [16, 64])
def test_sharp_rows_and_the_same_bits_in_large_workgroups(new, lens, heads, heads_kv, d, dtype, page):
    """Queries 30 times as large: a row's reference moves often, and by much more than the 2^8 it may lag behind."""
    b = Batch(new, lens, heads, heads_kv, d, dtype, page, gain=30.0, seed=42)
    O, lse = b.attend()
    b.check(O, lse)
    other = torch.empty((4096, 4096), device=O.device)
    for k in range(6):
        if k % 2:                                              # next to other work
            with torch.cuda.stream(torch.cuda.Stream()):
                other.normal_()
        O2, lse2 = b.attend()
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
