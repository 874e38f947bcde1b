"""Pins of the 64-bit oracle of the cache of pages: against the framework's other oracles and closed forms.  CPU only."""
import numpy as np
import pytest
import torch

import oracle as orc
import oracle.paged as paged


def test_a_grid_of_adjacent_pairs_is_the_table_oracle():
    frames, h, w, pairs, d = [2, 3, -1], 3, 4, (12, 10, 10), 64
    n = len(frames) * h * w
    cos, sin = orc.rope_tables_3d(np.array(frames), h, w, pairs)
    x = np.random.default_rng(0).standard_normal((n, d))
    t = np.arange(n)
    pos = np.stack([np.array(frames)[t // (h * w)], t // w % h, t % w])
    got = paged.rotate_axes(x, pos, pairs, halves=False, shared=False)
    assert np.abs(got - orc.rope_rotate(x, cos, sin)).max() < 1e-13


@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("shared", [True, False])
def test_inner_products_follow_the_distance_alone(halves, shared):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 32))
    pairs, at = [5, 4, 3], np.array([[7], [3], [11]])
    turn = lambda x, p: paged.rotate_axes(x, p, pairs, halves=halves, shared=shared)  # noqa: E731
    near = turn(q, at) @ turn(k, at + np.array([[2], [-1], [5]])).T
    far = turn(q, at + 1000) @ turn(k, at + 1000 + np.array([[2], [-1], [5]])).T
    assert abs(float((near - far).item())) < 1e-10
    back = paged.rotate_axes(turn(q, at), at, pairs, halves=halves, shared=shared, inverse=True)
    assert np.abs(back - q).max() < 1e-14 and np.array_equal(turn(q, at)[:, 24:], q[:, 24:])


def _pages(keys, values, page, rng):
    n, Hk, d = keys.shape
    count = -(-n // page)
    K, V = rng.standard_normal((2, count + 1, Hk, page, d))
    table = rng.permutation(count + 1)[:count][None]
    return *paged.append(K, V, keys, values, [0, n], [n], table), table


@pytest.mark.parametrize("causal,window,sink", [(True, 0, 0), (False, 0, 0), (True, 7, 0), (True, 5, 3), (False, 9, 2)])
def test_attention_is_the_librarys_on_a_mask_written_out(causal, window, sink):
    rng = np.random.default_rng(2)
    n, m, H, Hk, d, page = 41, 13, 6, 2, 16, 5
    keys, values = rng.standard_normal((2, n, Hk, d))
    K, V, table = _pages(keys, values, page, rng)
    Q = rng.standard_normal((m, H, d))
    O, lse2, spread, _, count = paged.attend(Q, K, V, [0, m], [n], table, causal, window, sink)
    mask = np.zeros((m, n), dtype=bool)
    for i in range(m):
        for j in range(n):
            p = n - m + i
            mask[i, j] = (not causal or j <= p) and (not window or j > p - window or j < sink)
    t = lambda x: torch.tensor(np.ascontiguousarray(x.transpose(1, 0, 2)))  # noqa: E731
    ref = torch.nn.functional.scaled_dot_product_attention(t(Q), t(keys).repeat_interleave(3, 0), t(values).repeat_interleave(3, 0),
                                                           attn_mask=torch.tensor(mask))
    assert np.abs(O.transpose(1, 0, 2) - ref.numpy()).max() < 1e-12 and np.array_equal(count, mask.sum(1))
    logit = np.einsum("mhd,nhd->hmn", Q, np.repeat(keys, 3, 1)) / 4.0
    lse = np.log(np.where(mask, np.exp(logit), 0.0).sum(-1)) / np.log(2.0)
    assert np.abs(lse2 - lse).max() < 1e-12 and (spread >= np.abs(O) - 1e-12).all()


def test_dense_window_attention_is_the_same_thing():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 24, 1, 32))
    K, V, table = _pages(k, v, 7, rng)
    O, *_ = paged.attend(q, K, V, [0, 24], [24], table, causal=False)
    assert np.abs(O[:, 0] - orc.dense_attention(q[:, 0], k[:, 0], v[:, 0])).max() < 1e-12


def test_rows_without_a_key_and_pages_that_are_none():
    rng = np.random.default_rng(4)
    K, V = rng.standard_normal((2, 3, 1, 4, 8))
    Q = rng.standard_normal((5, 1, 8))
    table = np.array([[0, 7], [-1, 2]])
    O, lse2, _, _, count = paged.attend(Q, K, V, [0, 3, 4], [1, 4], table)
    assert list(count) == [0, 0, 1, 0, 0] and np.array_equal(O[2, 0], V[0, 0, 0])
    assert np.isinf(lse2[0, [0, 1, 3]]).all() and (O[[0, 1, 3]] == 0).all() and np.isnan(O[4]).all()
