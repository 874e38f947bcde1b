"""Attention over several caches joined by lse2, as the header has it; against the 64-bit oracle over all keys."""
import numpy as np
import pytest
import torch

from paged import HALF, Batch, f64

pytestmark = pytest.mark.gpu


def _join(parts):
    """Parts (O, lse2 [heads, rows]) -> O in 64 bits: weights 2^(lse2 - the largest), +inf is a part without a key."""
    lse = np.stack([f64(lse2).T for _, lse2 in parts])                                   # [parts, rows, heads]
    empty = np.isposinf(lse)
    top = np.where(empty, -np.inf, lse).max(0)
    w = np.where(empty, 0.0, np.exp2(np.where(empty, 0.0, lse) - np.where(np.isinf(top), 0.0, top)))
    total = w.sum(0)
    O = sum(x[..., None] * f64(o) for x, (o, _) in zip(w, parts))
    return O / np.where(total > 0, total, 1.0)[..., None]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1, 1, 1, 1], [40, 1, 3, 130, 2, 7]])
def test_parts_over_two_caches(dtype, d, new):
    """Every sequence's first pages in one cache, the others in another; some sequences have none in one of them, one has none in both."""
    page, first = 16, [3, 0, 2, 1, 40, 0]               # pages in the first cache
    lens = [100, 60, 32, 17, 1000, 0]
    whole = Batch(new, lens, 6, 2, d, dtype, page, causal=False, seed=40)
    ref = whole.oracle()
    table, parts = whole.table.copy(), []
    for second in (False, True):
        part = Batch(new, lens, 6, 2, d, dtype, page, causal=False, seed=40)
        for s, k in enumerate(first):
            row = table[s, k:] if second else table[s, :k]
            part.table[s] = -1
            part.table[s, :len(row)] = row
            part.lens[s] = max(0, lens[s] - k * page) if second else min(lens[s], k * page)
        part.to_gpu()
        O, lse2 = part.attend()
        part.check(O, lse2)
        assert np.isposinf(f64(lse2)).any() and np.isfinite(f64(lse2)).any()
        parts.append((O, lse2))
    got = _join(parts)
    assert np.isfinite(got).all()
    # the bounds of tests/paged.py, once more a rounding of each part's output, and weights that are off by ln 2 of what their lse2 is
    R, L, spread, size, count = ref
    delta = (d + 8) * 2.0 ** -24 * size[..., None]
    sums = (count[:, None, None] + 64) * 2.0 ** -24
    lse_off = 1.5 * (delta + 2 * sums) + 2.0 ** -22 * np.abs(np.where(np.isinf(L), 0.0, L)).max(0)[:, None, None]
    part_off = (HALF["bf16"] if dtype == "bf16" else 0.0) + HALF[dtype] + 2 * delta + 2 * sums
    bound = spread * (part_off + 2 * np.log(2.0) * 1.01 * lse_off)
    assert (np.abs(got - R) <= bound).all(), (np.abs(got - R) - bound).max()
    assert (got[count == 0] == 0).all() and (count == 0).any()
