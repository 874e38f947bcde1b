"""The cache of pages: new tokens enter it, and attention reads it; against the 64-bit oracle, element by element (bounds: tests/paged.py)."""
import numpy as np
import pytest
import torch

import oracle.paged as orc
import paper_2604_10103_amd as hf
from paged import DEV, TYPES, Batch, f64

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 7, 16, 40])
@pytest.mark.parametrize("form", ["plain", "place", "adjacent", "halves", "odd"])
def test_appended_tokens_lie_in_their_pages(dtype, d, page, form):
    new, lens = [1, 0, 5, 33, 1, 3], [1, 9, 5, 70, 17, 2]     # the last one's first token lies before the sequence
    b = Batch(new, lens, 6, 2, d, dtype, page, rows_behind=4, seed=page + d)
    b.table[2, 0] = b.n_pages + 3                              # no page: dropped
    b.to_gpu()
    pairs = {"plain": None, "place": [d // 2], "adjacent": [d // 2 - 2 * (d // 6), d // 6, d // 6], "halves": [d // 4, d // 8, d // 8],
             "odd": [5, 4]}[form]
    rope = pos = None
    if pairs:
        rope = hf.make_rope_axes(pairs, layout=hf.HF_ROPE_ADJACENT if form == "adjacent" else hf.HF_ROPE_HALVES)
        if form != "place":
            pos = torch.randint(0, 900, (len(pairs), b.n), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(DEV)
    places = np.concatenate([np.arange(n - m, n) for m, n in zip(new, lens)] + [np.zeros(4, dtype=int)])
    turned = {}
    for name, x in (("K", b.K), ("Q", b.Q)):
        if pairs:   # what hf_rope_axes_apply writes, to the bit
            y = torch.empty((b.n, x.shape[1], d), dtype=b.t, device=DEV)
            p = pos if pos is not None else torch.tensor(places, dtype=torch.int32, device=DEV)[None]
            hf.hf_rope_axes_apply(rope, x, p, y)
            turned[name] = y
        else:
            turned[name] = x.clone()
    want_K, want_V = orc.append(f64(b.K_pages), f64(b.V_pages), f64(turned["K"]), f64(b.V), b.cu, b.lens, b.table)
    keep_K, keep_V = b.K_pages.clone(), b.V_pages.clone()
    Q_out = torch.full((b.n, 6, d), 7.0, dtype=b.t, device=DEV)
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d, rope=rope, positions=pos, Q=b.Q, Q_out=Q_out)
    assert np.array_equal(f64(b.K_pages), want_K) and np.array_equal(f64(b.V_pages), want_V)
    assert torch.equal(Q_out[:-4], turned["Q"][:-4]) and (Q_out[-4:] == 7.0).all()
    # without queries, and with queries turned where they lie
    b.K_pages.copy_(keep_K)
    b.V_pages.copy_(keep_V)
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d, rope=rope, positions=pos)
    assert np.array_equal(f64(b.K_pages), want_K) and np.array_equal(f64(b.V_pages), want_V)
    K, V = b.K.clone(), b.V.clone()
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d, rope=rope, positions=pos, Q=b.Q, Q_out=b.Q)
    assert torch.equal(b.Q[:-4], turned["Q"][:-4]) and torch.equal(b.K, K) and torch.equal(b.V, V)


def test_many_sequences_find_their_rows():
    rng = np.random.default_rng(0)
    new = rng.choice([0, 1, 1, 2, 5], size=700)
    lens = new + rng.integers(0, 20, size=700)
    b = Batch(new, lens, 2, 1, 64, "bf16", 16, seed=3)
    want_K, want_V = orc.append(f64(b.K_pages), f64(b.V_pages), f64(b.K), f64(b.V), b.cu, b.lens, b.table)
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d)
    assert np.array_equal(f64(b.K_pages), want_K) and np.array_equal(f64(b.V_pages), want_V)


def test_values_that_are_copied_keep_every_bit():
    b = Batch([3], [3], 1, 1, 64, "bf16", 4)
    bits = torch.randint(-32768, 32767, (3, 1, 64), generator=torch.Generator().manual_seed(2), dtype=torch.int32).to(torch.int16).to(DEV)
    V = bits.view(torch.bfloat16)                              # NaNs of every kind among them
    hf.hf_paged_append(b.cache, b.K, V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d, rope=hf.make_rope_axes([32]))
    assert torch.equal(b.V_pages[int(b.table[0, 0])].transpose(0, 1)[:3].view(torch.int16), bits)


# ---------------------------------------------------------------------------------------------------- attention
MASKS = [dict(), dict(causal=False), dict(window=9), dict(window=30, n_sink=3), dict(causal=False, window=50, n_sink=17),
         dict(window=1), dict(causal=False, window=5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", MASKS)
def test_single_tokens(dtype, d, mask):
    lens = [1, 2, 31, 32, 33, 0, 64, 65, 200, 517, 1000]
    b = Batch([1] * len(lens), lens, 8, 2, d, dtype, 16, seed=d, **mask)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", MASKS)
def test_chunks_and_single_tokens_in_one_batch(dtype, d, mask):
    new, lens = [40, 1, 0, 17, 130, 3], [40, 77, 12, 300, 131, 3]
    b = Batch(new, lens, 6, 2, d, dtype, 40, rows_behind=5, seed=d + 1, **mask)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 2, 3, 8, 15, 16, 24, 31, 32, 33, 100, 128, 1560])
def test_pages_of_any_size(dtype, page):
    b = Batch([1, 45, 2], [97, 150, 1], 4, 2, 128, dtype, page, seed=page)
    b.check(*b.attend())
    b = Batch([5, 1], [150, 33], 4, 2, 64, dtype, page, causal=False, window=70, n_sink=5, seed=page)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [94, 256, 300, 500, 1000])
@pytest.mark.parametrize("mask", [dict(), dict(causal=False, window=400, n_sink=70), dict(window=333, n_sink=95)])
def test_long_pages_end_inside_a_tile(dtype, page, mask):
    b = Batch([1, 290, 2], [1300, 1290, 501], 4, 2, 128, dtype, page, seed=page, **mask)
    b.check(*b.attend())
    b = Batch([1, 3], [1300, 999], 4, 1, 64, dtype, page, seed=page, **mask)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64, 94])
def test_pages_that_are_none_inside_long_contexts(dtype, page):
    b = Batch([1, 200, 40], [1300, 700, 41], 4, 2, 128, dtype, page, seed=page)
    b.table[0, 3] = b.table[0, 5] = -5
    b.table[1, 2] = b.n_pages
    b.table[1, 5] = 2 ** 31 - 1
    b.table[2, 0] = -1
    b.to_gpu()
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,heads_kv", [(1, 1), (3, 3), (5, 1), (16, 1), (33, 1), (70, 2), (40, 8), (12, 12)])
def test_groups_of_heads(dtype, heads, heads_kv):
    b = Batch([1, 2, 9], [40, 100, 9], heads, heads_kv, 64, dtype, 16, seed=heads)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_long_contexts_are_shared_out(dtype, d):
    """Enough keys that several workgroups share a row's."""
    b = Batch([1, 2, 1], [20000, 9001, 5], 4, 2, d, dtype, 64, seed=7)
    b.check(*b.attend())
    b = Batch([150], [6000], 2, 1, d, dtype, 64, seed=8)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gain", [30.0])
def test_sharp_softmax_rescales(dtype, gain):
    b = Batch([1, 60, 1], [700, 333, 3000], 4, 2, 128, dtype, 32, gain=gain, seed=9)
    b.check(*b.attend())


@pytest.mark.parametrize("scale", [0.25, 1e-3])
def test_softmax_scale(scale):
    b = Batch([1, 20], [90, 50], 4, 4, 64, "bf16", 16, scale=scale, seed=10)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_key(dtype):
    """New tokens before the sequence (more of them than its length), empty sequences, pages that are none."""
    b = Batch([6, 1, 2, 40], [3, 0, 40, 40], 4, 2, 64, dtype, 8, rows_behind=3, seed=11, extra_entries=1)
    b.table[2, :] = -1
    b.table[3, 1] = b.n_pages
    b.table[3, 3] = -(2 ** 31)
    b.to_gpu()
    b.check(*b.attend())
    b.cache.causal = 0
    b.mask["causal"] = False
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("mask", [dict(), dict(window=20, n_sink=4), dict(causal=False)])
@pytest.mark.parametrize("new,n", [(70, 70), (150, 200), (3, 90), (1, 64)])
@pytest.mark.parametrize("page", [24, 64, 94])
def test_what_is_not_seen_does_not_count(dtype, d, bad, mask, new, n, page):
    """Keys and values that are not finite reach the rows that see them and no others, beyond the length included."""
    b = Batch([new, 1], [n, 50], 4, 2, d, dtype, page, seed=12, **mask)
    b.check(*b.attend())
    ref = b.oracle()
    clean, clean_lse = b.attend()
    where = [j for j in {n - 1, n - new + new // 2, n - new // 3, max(0, n - 40)} if 0 <= j < n]
    for pages in (b.K_pages, b.V_pages):
        for j in where:
            pages[int(b.table[0, j // page]), :, j % page, :5] = bad
        for s, length in ((0, n), (1, 50)):                    # what lies behind the length in its last page
            if length % page:
                pages[int(b.table[s, length // page]), :, length % page:] = bad
        for spare in set(range(b.n_pages)) - set(b.table.flatten().tolist()):
            pages[spare] = bad
    O, lse = b.attend()
    hit = np.zeros(b.n, dtype=bool)
    for i in range(new):
        seen = orc.sees(n - new + i, n, **b.mask)
        hit[i] = any(seen[j] for j in where)
    untouched = torch.tensor(~hit, device=DEV)
    assert torch.equal(O[untouched], clean[untouched]) and torch.equal(lse[:, untouched], clean_lse[:, untouched])
    if hit.any():
        # a key that is not finite gives NaN, +inf or -inf as a score: in the rows that see it nothing can be asserted but that a NaN
        # key makes the whole row NaN
        rows = torch.tensor(hit, device=DEV)
        if bad != bad:
            assert torch.isnan(O[rows]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("page", [24, 32, 94])
def test_values_that_are_not_finite_reach_their_features(dtype, d, bad, page):
    """Values alone: a visible one makes its own feature NaN or that infinity, the others stay within their bounds."""
    new, n = 100, 140
    b = Batch([new], [n], 4, 2, d, dtype, page, window=50, n_sink=2, seed=13)
    ref = b.oracle()
    where = {90: 3, 120: d - 1, 139: 17, 45: 40}
    for j, f in where.items():
        b.V_pages[int(b.table[0, j // page]), :, j % page, f] = bad
    O, lse = b.attend()
    got, fine = f64(O), np.ones((new, d), dtype=bool)
    for i in range(new):
        seen = orc.sees(n - new + i, n, **b.mask)
        for j, f in where.items():
            if seen[j]:
                fine[i, f] = False
                assert all(np.isnan(x) if bad != bad else (x == bad or np.isnan(x)) for x in got[i, :, f])
    for h in range(4):
        o, r = got[:, h][fine], ref[0][:, h][fine]
        assert np.isfinite(o).all() and np.abs(o - r).max() <= (2e-2 if dtype == "bf16" else 1e-5) * np.abs(ref[2]).max()
    b.check(torch.tensor(np.where(fine[:, None], got, ref[0]), device=DEV), lse, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,longest", [([0, 1, 1, 2, 5], 200), ([0, 1, 60, 90], 300)])
@pytest.mark.parametrize("heads,heads_kv,d", [(4, 2, 64), (8, 4, 64), (4, 4, 128)])
def test_more_sequences_than_a_wavefront_has_lanes(dtype, new, longest, heads, heads_kv, d):
    rng = np.random.default_rng(len(new))
    new = rng.choice(new, size=300)
    b = Batch(new, new + rng.integers(0, longest, size=300), heads, heads_kv, d, dtype, 16, rows_behind=2, seed=20)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,count", [(128, 16, 72), (64, 94, 72), (64, 40, 20), (128, 16, 300), (64, 94, 300)])
def test_long_sequences_of_single_tokens(dtype, d, page, count):
    """More keys than one round of workgroups takes, of sequences that differ: a workgroup has several sequences, and parts of some."""
    rng = np.random.default_rng(count)
    lens = rng.integers(1, 72 * 2500 // count, size=count)
    lens[3], lens[7] = 0, 1
    new = rng.choice([1, 1, 1, 3], size=count)
    b = Batch(new, lens, 8, 4, d, dtype, page, seed=21)
    ref = b.oracle()
    O, lse = b.attend()
    b.check(O, lse, ref)
    O2, lse2 = b.attend()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    b = Batch(new, lens, 8, 4, d, dtype, page, seed=22, window=1200, n_sink=50)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("short,count,heads", [(96, 110, 8), (64, 118, 8), (32, 100, 8), (20, 300, 4), (96, 300, 4)])
def test_short_sequences_end_where_a_share_does(dtype, d, short, count, heads):
    """Short sequences between long ones: workgroups' shares of the work end at, before and behind the ends of the short ones."""
    lens = np.full(count, short)
    lens[::2] = 1024
    b = Batch([1] * count, lens, heads, heads, d, dtype, 16, seed=31)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(window=900, n_sink=40), dict(causal=False, window=900, n_sink=40)])
@pytest.mark.parametrize("count,new,page", [(100, [0, 0, 0, 1, 3, 260], 16), (70, [0, 0, 1, 40, 700], 64), (90, [0, 1, 1, 2], 64)])
def test_parts_of_many_sequences(dtype, mask, count, new, page):
    """More sequences than a wavefront has lanes, few rows, long contexts: chunks and single tokens of some of them come in parts."""
    rng = np.random.default_rng(count)
    new = rng.choice(new, size=count)
    lens = new + rng.integers(0, 3500, size=count) * (rng.random(count) < 0.3)
    b = Batch(new, lens, 2, 1, 64, dtype, page, seed=32, **mask)
    b.check(*b.attend())


@pytest.mark.parametrize("page", [24, 64])
@pytest.mark.parametrize("mask", [dict(), dict(causal=False, window=700, n_sink=64), dict(window=500)])
def test_long_chunks_of_many_heads(page, mask):
    b = Batch([1030, 5, 131], [1300, 400, 131], 32, 32, 128, "bf16", page, seed=23, **mask)
    b.check(*b.attend())


@pytest.mark.parametrize("heads,heads_kv,new,lens", [(4, 1, [900], [900]), (8, 2, [700, 300], [2500, 300]), (2, 2, [1500, 1, 40], [1500, 6000, 3000])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 600])
def test_long_causal_chunks_of_few_heads(dtype, heads, heads_kv, new, lens, window):
    """Few rows for the chip: row tiles have parts, the later ones more of them."""
    b = Batch(new, lens, heads, heads_kv, 64, dtype, 32, seed=24, window=window, n_sink=window // 50)
    b.check(*b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_past_32_bits(dtype):
    """Pages on both sides of every 4 GiB of the pools, written by the append and read by both shapes of attention."""
    page, Hk, d = 64, 8, 128
    size = Hk * page * d * (2 if dtype == "bf16" else 4)
    n_pages = (9 << 30) // size + 3
    b = Batch([1, 200, 3], [300, 200, 130], 8, Hk, d, dtype, page, seed=25)
    used = [int(x) for x in b.table.flatten() if x >= 0]
    edge = (4 << 30) // size
    far = [0, edge - 1, edge, edge + 1, 2 * edge - 1, 2 * edge, 2 * edge + 1, n_pages - 1, n_pages - 2, n_pages - 3, 1, 5, 7]
    assert len(used) <= len(far)
    K, V = torch.empty((n_pages, Hk, page, d), dtype=b.t, device=DEV), torch.empty((n_pages, Hk, page, d), dtype=b.t, device=DEV)
    move = dict(zip(used, far))
    for x, y in move.items():
        K[y], V[y] = b.K_pages[x], b.V_pages[x]
    small, cache, table = (b.K_pages, b.V_pages), b.cache, b.table_d
    want_K, want_V = orc.append(f64(b.K_pages), f64(b.V_pages), f64(b.K), f64(b.V), b.cu, b.lens, b.table)
    big = hf.make_paged(8, Hk, d, dtype, page, n_pages, 3, b.table.shape[1])
    far_table = torch.tensor(np.vectorize(lambda x: move.get(x, -1))(b.table), dtype=torch.int32, device=DEV)
    hf.hf_paged_append(big, b.K, b.V, b.cu_d, b.lens_d, K, V, far_table)
    for x, y in move.items():
        assert np.array_equal(f64(K[y]), want_K[x]) and np.array_equal(f64(V[y]), want_V[x])
    hf.hf_paged_append(cache, b.K, b.V, b.cu_d, b.lens_d, *small, table)
    ref = b.oracle()
    O, lse = b.attend()
    b.check(O, lse, ref)
    for count in (1, 3):   # the single token alone, and the whole batch
        n = int(b.cu[count])
        c = hf.make_paged(8, Hk, d, dtype, page, n_pages, count, b.table.shape[1])
        ws = torch.empty(max(1, hf.hf_paged_workspace_bytes(c, n)), dtype=torch.uint8, device=DEV)
        out = torch.empty((n, 8, d), dtype=b.t, device=DEV)
        hf.hf_paged_attn_fwd(c, b.Q[:n], b.cu_d[:count + 1], b.lens_d[:count], K, V, far_table[:count], out, ws)
        b.check(torch.cat([out, O[n:]]), None, ref)


def test_the_same_bits_every_time_and_in_any_workspace():
    b = Batch([1] * 30 + [70], list(range(1, 6000, 200)) + [900], 8, 2, 128, "bf16", 16, seed=14)
    O, lse = b.attend()
    n = max(1, hf.hf_paged_workspace_bytes(b.cache, b.n))
    for fill in (0, 255, 1):
        O2, lse2 = b.attend(workspace=torch.full((n,), fill, dtype=torch.uint8, device=DEV))
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    for _ in range(5):   # the same workspace again and again
        O2, lse2 = b.attend(workspace=ws)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)


def test_sequences_share_pages_and_come_in_any_order():
    b = Batch([4, 4, 4], [100, 100, 100], 4, 2, 64, "bf16", 16, seed=15)
    b.table[1, :6] = b.table[0, :6]                            # a common beginning of 96 tokens
    b.table[2] = b.table[0]
    b.to_gpu()
    b.check(*b.attend())


def test_strided_operands():
    b = Batch([3, 40, 1], [30, 60, 200], 6, 3, 128, "bf16", 16, seed=16)
    want, _ = b.attend()
    wide = torch.full((6, b.n, 136), 7.0, dtype=torch.bfloat16, device=DEV)
    O, _ = b.attend(O=wide[:, :, :128].transpose(0, 1))
    assert torch.equal(O, want) and (wide[:, :, 128:] == 7.0).all()
    b.Q = b.Q.transpose(0, 1).contiguous().transpose(0, 1)
    O, _ = b.attend()
    assert torch.equal(O, want)


def test_another_stream():
    b = Batch([1, 50], [3000, 400], 8, 2, 128, "bf16", 16, seed=17)
    want, lse = b.attend()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        O, lse2 = b.attend()
    s.synchronize()
    assert torch.equal(O, want) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_captured_calls_share_a_workspace(dtype):
    """Replays in turn, with eager calls in the same workspace and other lengths in between; every one against an eager call of its own."""
    a = Batch([1] * 9, [5000, 3, 700, 64, 1, 2500, 33, 900, 4000], 8, 2, 128, dtype, 16, seed=26)
    b = Batch([150, 3], [6000, 2000], 8, 2, 128, dtype, 64, seed=27)
    n = max(hf.hf_paged_workspace_bytes(x.cache, x.n) for x in (a, b))
    ws = torch.randint(0, 255, (n,), dtype=torch.uint8, device=DEV)
    outs, graphs = [], []
    full = [x.lens_d.clone() for x in (a, b)]
    for x in (a, b):
        x.lens_d.copy_(torch.clamp(x.lens_d, max=40))          # captured with other lengths than replayed
        O, lse = torch.empty((x.n, 8, 128), dtype=x.t, device=DEV), torch.empty((8, x.n), device=DEV)
        run = lambda x=x, O=O, lse=lse: hf.hf_paged_attn_fwd(x.cache, x.Q, x.cu_d, x.lens_d, x.K_pages, x.V_pages, x.table_d, O, ws, lse)  # noqa: E731
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        outs.append((O, lse))
        graphs.append((g, run))
    for x, n in zip((a, b), full):
        x.lens_d.copy_(n)
    want = [x.attend() for x in (a, b)]
    for x, w in zip((a, b), want):
        x.check(*w)
    for k in range(6):
        for i in (0, 1):
            outs[i][0].fill_(3.0)
            graphs[i][0].replay()
            if k % 2:
                torch.cuda.synchronize()
            assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
        if k == 2:
            graphs[0][1]()                                     # eager, in the same workspace
            assert torch.equal(outs[0][0], want[0][0])
    a.lens_d.copy_(torch.tensor([1, 2, 5000, 0, 60, 61, 62, 63, 64], dtype=torch.int32))
    a.lens = a.lens_d.cpu().numpy().astype(np.int64)
    a.table[2] = a.table[0]                                    # the third sequence is as long as the first was
    a.table_d.copy_(torch.tensor(a.table, dtype=torch.int32))
    graphs[0][0].replay()
    a.check(outs[0][0], None)


def test_calls_on_several_streams_at_once():
    batches = [Batch([1] * 20, list(range(10, 4010, 200)), 8, 2, 128, "bf16", 16, seed=28), Batch([300], [3000], 4, 2, 64, "bf16", 32, seed=29),
               Batch([2, 1], [9000, 50], 8, 2, 64, "f32", 16, seed=30)]
    want = [b.attend() for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[] for _ in batches]
    spaces = [b.workspace() for b in batches]
    torch.cuda.synchronize()
    for _ in range(8):
        for i, (b, s) in enumerate(zip(batches, streams)):
            with torch.cuda.stream(s):
                got[i].append(b.attend(workspace=spaces[i]))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(O, w[0]) and torch.equal(lse, w[1]) for O, lse in g)


def test_no_rows():
    b = Batch([0, 0], [5, 9], 4, 2, 64, "bf16", 16)
    O, lse = b.attend()
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.table_d)


# ---------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal,window,sink,page,pairs,halves", [(True, 0, 0, 16, [64], True), (False, 90, 30, 30, [22, 21, 21], False)])
def test_sequences_grow_step_by_step(dtype, causal, window, sink, page, pairs, halves):
    """Prompts (or chunks of frames), then single tokens, in one captured step for all of them: every step against attention over the
    whole history, rotated by the oracle."""
    S, H, Hk, d, steps = 3, 4, 2, 128, 5
    first = [37, 1, 64]
    b = Batch(first, first, H, Hk, d, dtype, page, causal=causal, window=window, n_sink=sink, seed=18)
    width = -(-(max(first) + steps) // page)
    b.n_pages = S * width
    b.table = np.random.default_rng(1).permutation(b.n_pages).reshape(S, width).astype(np.int32)
    b.K_pages = torch.full((b.n_pages, Hk, page, d), float("nan"), dtype=b.t, device=DEV)
    b.V_pages = b.K_pages.clone()
    cache = hf.make_paged(H, Hk, d, dtype, page, b.n_pages, S, width, causal=causal, window=window, n_sink=sink)
    rope = hf.make_rope_axes(pairs, layout=hf.HF_ROPE_HALVES if halves else hf.HF_ROPE_ADJACENT)
    lens = torch.tensor(first, dtype=torch.int32, device=DEV)
    table = torch.tensor(b.table, device=DEV)
    history = [[] for _ in range(S)]

    def place(lens_now, counts):
        at = np.concatenate([np.arange(n - m, n) for n, m in zip(lens_now, counts)])
        return np.stack([at // (1 + 3 * a) for a in range(len(pairs))])

    def check(rows, O, cu, lens_now, pos):
        q = orc.rotate_axes(f64(rows[:, :H]).transpose(1, 0, 2), pos, pairs, halves=halves).transpose(1, 0, 2)
        k = orc.rotate_axes(f64(rows[:, H:H + Hk]).transpose(1, 0, 2), pos, pairs, halves=halves).transpose(1, 0, 2)
        v = f64(rows[:, H + Hk:])
        for s in range(S):
            for i in range(cu[s], cu[s + 1]):
                history[s].append((k[i], v[i]))
        for s in range(S):
            K, V = np.stack([x[0] for x in history[s]]), np.stack([x[1] for x in history[s]])
            for i in range(cu[s], cu[s + 1]):
                ok = orc.sees(lens_now[s] - cu[s + 1] + i, lens_now[s], causal, window, sink)
                for h in range(H):
                    logit = K[ok, h // 2] @ q[i, h] / np.sqrt(d)
                    w = np.exp(logit - logit.max())
                    ref = w @ V[ok, h // 2] / w.sum()
                    # rounding of rotated q and k moves a logit by 2 half steps of |q| |k| sizes; then as a bound of tests/paged.py
                    size = (np.abs(K[ok, h // 2]) @ np.abs(q[i, h])).max() / np.sqrt(d)
                    half = 2.0 ** -8 if dtype == "bf16" else 6 * 2.0 ** -24
                    spread = w @ np.abs(V[ok, h // 2]) / w.sum()
                    assert (np.abs(f64(O[i, h]) - ref) <= half * np.abs(ref) + spread * (half + 4 * half * size + 1e-5)).all()

    ws = torch.empty(max(1, hf.hf_paged_workspace_bytes(cache, b.n)), dtype=torch.uint8, device=DEV)
    O = torch.empty((b.n, H, d), dtype=b.t, device=DEV)
    Q = torch.empty_like(O)
    pos = place(first, first)
    hf.hf_paged_append(cache, b.K, b.V, b.cu_d, lens, b.K_pages, b.V_pages, table, rope=rope,
                       positions=torch.tensor(pos, dtype=torch.int32, device=DEV), Q=b.Q, Q_out=Q)
    hf.hf_paged_attn_fwd(cache, Q, b.cu_d, lens, b.K_pages, b.V_pages, table, O, ws)
    check(b.rows, O, b.cu, first, pos)
    # one token each, captured: lengths, positions and tokens are what changes
    rows = torch.empty((S, H + 2 * Hk, d), dtype=b.t, device=DEV)
    pos_d, cu = torch.zeros((len(pairs), S), dtype=torch.int32, device=DEV), torch.arange(S + 1, dtype=torch.int32, device=DEV)
    q1, O1 = torch.empty((S, H, d), dtype=b.t, device=DEV), torch.empty((S, H, d), dtype=b.t, device=DEV)
    ws1 = torch.empty(max(1, hf.hf_paged_workspace_bytes(cache, S)), dtype=torch.uint8, device=DEV)

    def step():
        hf.hf_paged_append(cache, rows[:, H:H + Hk], rows[:, H + Hk:], cu, lens, b.K_pages, b.V_pages, table, rope=rope, positions=pos_d,
                           Q=rows[:, :H], Q_out=q1)
        hf.hf_paged_attn_fwd(cache, q1, cu, lens, b.K_pages, b.V_pages, table, O1, ws1)

    g, now = None, list(first)
    for k in range(steps):
        rows.copy_(torch.randn(rows.shape, generator=torch.Generator().manual_seed(100 + k)).to(b.t))
        now = [n + 1 for n in now]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        pos = place(now, [1] * S)
        pos_d.copy_(torch.tensor(pos, dtype=torch.int32))
        if k == 0:
            step()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        else:
            g.replay()
        torch.cuda.synchronize()
        check(rows, O1, list(range(S + 1)), now, pos)
