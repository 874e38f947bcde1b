"""New tokens enter pages in 8 bits: against the 64-bit oracle, and to the bit where nothing is computed before the rounding."""
import numpy as np
import pytest
import torch

import oracle.e4m3 as orc
import oracle.paged as paged
import paper_2604_10103_amd as hf
from e4m3 import UNIT, Batch8, norm_bound, rope_of, values
from paged import DEV, f64
from test_gpu_norm_rope import _form

pytestmark = pytest.mark.gpu

NEW, LENS = [1, 0, 5, 33, 1, 3], [1, 9, 5, 70, 17, 2]     # the last one's first token lies before the sequence


def _append(b, q=True, **how):
    out = torch.full((b.n, b.heads, b.d), 7.0, dtype=b.t, device=DEV)
    hf.hf_paged_append_e4m3(b.cache, b.K, b.V, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.K_scales, b.V_scales, b.table_d,
                            Q=b.Q if q else None, Q_out=out if q else None, **how)
    return out


def _slots(b):
    """(row, page, place) of every row that has a slot."""
    out = []
    for s, (m, n) in enumerate(zip(NEW, b.lens)):
        for i in range(m):
            j = int(n) - m + i
            if 0 <= j < b.table.shape[1] * b.page and 0 <= b.table[s, j // b.page] < b.n_pages:
                out.append((int(b.cu[s]) + i, int(b.table[s, j // b.page]), j % b.page))
    return out


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 7, 16, 40])
@pytest.mark.parametrize("form", ["alone", "adjacent", "halves", "axes", "odd", "place"])
@pytest.mark.parametrize("weights", ["none", "one", "each"])
def test_appended_rows(dtype, d, page, form, weights):
    b = Batch8(NEW, LENS, 6, 2, d, dtype, page, rows_behind=4, seed=page + d)
    b.table[2, 0] = b.n_pages + 3                              # no page: dropped
    b.to_gpu()
    own, ref = _form("halves" if form == "place" else form, d)
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(0, 900, (len(ref["pairs"]), b.n), generator=g, dtype=torch.int32).to(DEV) if ref and form != "place" else None
    places = np.concatenate([np.arange(n - m, n) for m, n in zip(NEW, LENS)] + [np.zeros(4, dtype=int)])
    at = pos.cpu().numpy() if pos is not None else places[None]
    w = {"none": (None, None), "one": [torch.randn(d, generator=g).to(DEV) for _ in "kq"],
         "each": [torch.randn(h, d, generator=g).to(DEV) for h in (2, 6)]}[weights]
    eps = 1e-5
    before = [x.clone() for x in (b.K_pages.view(torch.uint8), b.V_pages.view(torch.uint8), b.K_scales, b.V_scales)]
    out = _append(b, norm=hf.make_head_norm(eps, weights == "each"), k_weight=w[0], q_weight=w[1], positions=pos, **own)
    how = lambda x: dict(weight=None if x is None else f64(x), eps=float(np.float32(eps)), positions=at if ref else None, **ref)  # noqa: E731
    live = sum(NEW)
    for name, rows, weight in (("Q", b.Q, w[1]), ("K", b.K, w[0])):
        x = f64(rows).transpose(1, 0, 2)
        y = orc.norm_turn(x, **how(weight))
        bound = norm_bound(x, "f32", y, **how(weight)).transpose(1, 0, 2)
        y = y.transpose(1, 0, 2)
        if name == "Q":
            far = np.abs(f64(out) - y) - norm_bound(x, dtype, y.transpose(1, 0, 2), **how(weight)).transpose(1, 0, 2)
            assert (far[:live] <= 0).all() and (f64(out)[live:] == 7.0).all()
            continue
        got, scale = values(b.K_pages, b.K_scales), f64(b.K_scales)
        for row, p, i in _slots(b):
            # the scale: the largest value's error, its constant's and its own rounding; a code: half its step, and the value's error
            s = scale[p, :, i]
            want = np.abs(y[row]).max(-1) / 448
            assert (np.abs(s - want) <= bound[row].max(-1) / 448 + 2 * UNIT * want).all()
            step = np.exp2(np.floor(np.log2(np.maximum(np.abs(got[p, :, i]) / s[:, None], 2.0 ** -6))) - 3) * s[:, None]
            # (where the value lies a hair above a power of two the code's own step is the larger one)
            assert (np.abs(got[p, :, i] - y[row]) <= 0.5 * step + bound[row] + 4 * UNIT * np.abs(y[row])).all()
    # values are quantised as they are: to the bit
    V = b.V.float().cpu()
    scale = torch.clamp(V.abs().amax(-1) * (1.0 / 448.0), min=2.0 ** -126)
    codes = (V / scale[..., None]).to(torch.float8_e4m3fn)
    want = [x.cpu().numpy().copy() for x in before]
    for row, p, i in _slots(b):
        want[1][p, :, i], want[3][p, :, i] = codes[row].view(torch.uint8).numpy(), scale[row].numpy()
    np.testing.assert_array_equal(_bytes(b.V_pages), want[1])
    np.testing.assert_array_equal(b.V_scales.cpu().numpy(), want[3])
    other = np.ones(b.K_scales.shape, dtype=bool)
    for _, p, i in _slots(b):
        other[p, :, i] = False
    np.testing.assert_array_equal(_bytes(b.K_pages)[other], want[0][other])
    np.testing.assert_array_equal(b.K_scales.cpu().numpy()[other], want[2][other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_only_quantised(dtype, d):
    """Neither norm nor rotation: keys and values to the bit, ties and the smallest and largest rows among them; queries are copied."""
    b = Batch8([200], [200], 4, 2, d, dtype, 32, seed=d)
    g = torch.Generator().manual_seed(d)
    x = torch.randint(-460, 460, (200, 8, d), generator=g) * torch.exp2(torch.randint(-20, 20, (200, 8, 1), generator=g).float())
    x[0], x[1, 4, 3], x[2, 6, 5], x[3, 5, 0] = 0.0, float("nan"), float("inf"), -float("inf")
    x[4:8] = torch.randn(4, 8, d, generator=g) * torch.tensor([2.0 ** -126, 2.0 ** -120, 2.0 ** 100, 2.0 ** 120])[:, None, None]
    x[8:40, :, 0] = 448.0                                     # a scale of (nearly) one: ties between codes
    x[8:40, :, 1:] = (torch.randint(-896, 896, (32, 8, d - 1), generator=g) / 2).clamp(-448, 448)
    x[40] *= torch.where(torch.rand(8, d, generator=g) < 0.3, -0.0, 1.0)
    b.rows.copy_(x.to(b.t))
    out = _append(b)
    assert torch.equal(_bytes_t(out), _bytes_t(b.Q))
    for rows, codes, scales in ((b.K, b.K_pages, b.K_scales), (b.V, b.V_pages, b.V_scales)):
        y = rows.float().cpu()
        bad = ~torch.isfinite(y).all(-1)
        scale = torch.clamp(y.abs().amax(-1) * (1.0 / 448.0), min=2.0 ** -126)
        want = torch.where(bad[..., None], 0, (y / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8))
        assert bad.any()
        place = torch.arange(200)
        page = torch.tensor(b.table[0])[place // 32].long()
        got, s = codes.view(torch.uint8).cpu()[page, :, place % 32], scales.cpu()[page, :, place % 32]
        assert torch.equal(torch.isnan(s), bad) and torch.equal(s[~bad], scale[~bad])
        assert torch.equal(got, want)


def _bytes_t(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("seqs", [1, 2, 33, 64, 65, 1000, 4097])
def test_many_sequences_find_their_rows(seqs):
    """Sequences of none, one or a few new tokens: every row lands in its own slot, whoever looks for it."""
    rng = np.random.default_rng(seqs)
    new = rng.choice([0, 0, 1, 1, 1, 2, 5], seqs)
    new[-1] = 1
    lens = new + rng.integers(0, 9, seqs)
    n, P = int(new.sum()), 8
    count = -(-np.maximum(lens, 1) // P)
    table = np.full((seqs, int(count.max())), -1, dtype=np.int32)
    order, at = rng.permutation(int(count.sum())), 0
    for s, k in enumerate(count):
        table[s, :k] = order[at:at + k]
        at += k
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    K = torch.randn(n, 1, 64, device=DEV).to(torch.bfloat16)
    cache = hf.make_paged(1, 1, 64, "bf16", P, at, seqs, table.shape[1])
    codes = [torch.zeros(at, 1, P, 64, dtype=torch.float8_e4m3fn, device=DEV) for _ in "kv"]
    scales = [torch.zeros(at, 1, P, device=DEV) for _ in "kv"]
    cu = np.concatenate([[0], np.cumsum(new)])
    hf.hf_paged_append_e4m3(cache, K, -K, ints(cu), ints(lens), *codes, *scales, ints(table))
    want = torch.zeros(at, P)
    scale = K.float().abs().amax(-1).cpu()[:, 0] * (1.0 / 448.0)
    for s in range(seqs):
        for i in range(int(new[s])):
            j = int(lens[s] - new[s] + i)
            want[table[s, j // P], j % P] = scale[cu[s] + i]
    for x in scales:
        assert torch.equal(x[:, 0].cpu(), want)


def test_pool_past_4_gib():
    """Places whose bytes do not fit in 32 bits."""
    P, Hk, d, pages = 1024, 4, 128, 9000                       # 4.7 GB of codes
    codes = [torch.zeros(pages, Hk, P, d, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in "kv"]
    scales = [torch.zeros(pages, Hk, P, device=DEV) for _ in "kv"]
    cache = hf.make_paged(Hk, Hk, d, "bf16", P, pages, 2, 1)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    K = torch.randn(6, Hk, d, device=DEV).to(torch.bfloat16)
    hf.hf_paged_append_e4m3(cache, K, -K, ints([0, 3, 6]), ints([P, P]), *codes, *scales, ints([[pages - 1], [pages - 2]]))
    for s, page in enumerate((pages - 1, pages - 2)):
        rows = K[3 * s:3 * s + 3].float().cpu().transpose(0, 1)
        scale = rows.abs().amax(-1) * (1.0 / 448.0)
        assert torch.equal(scales[0][page, :, -3:].cpu(), scale) and torch.equal(scales[1][page, :, -3:].cpu(), scale)
        want = (rows / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(codes[0][page, :, -3:].view(torch.uint8).cpu(), want)
    assert int((scales[0] != 0).sum()) == 24
    # and attention over them: the last row of each sees its own value
    Q = torch.randn(2, Hk, d, device=DEV).to(torch.bfloat16)
    O = torch.empty_like(Q)
    ws = torch.empty(hf.hf_paged_e4m3_workspace_bytes(cache, 2), dtype=torch.uint8, device=DEV)
    only = hf.make_paged(Hk, Hk, d, "bf16", P, pages, 2, 1, window=1)
    hf.hf_paged_attn_e4m3_fwd(only, Q, ints([0, 1, 2]), ints([P, P]), *codes, *scales, ints([[pages - 1], [pages - 2]]), O, ws)
    for s, page in enumerate((pages - 1, pages - 2)):
        v = codes[1][page, :, -1].float() * scales[1][page, :, -1, None]
        assert (O[s].float() - v).abs().le(v.abs() * 2.0 ** -6 + 1e-30).all()   # p v rounded, o rounded, and 1 / p


def test_places_agree_with_the_wide_cache():
    """The same batch into bf16 pages by hf_paged_append: the same slots, values as near as a code's half step."""
    b = Batch8([3, 17, 0, 1], [40, 17, 3, 64], 6, 3, 128, "bf16", 16, seed=4)
    rope = rope_of([64])
    out = _append(b, rope=rope)
    wide = torch.zeros(b.n_pages, 3, 16, 128, dtype=torch.bfloat16, device=DEV)
    wide_v, q = wide.clone(), torch.empty_like(out)
    hf.hf_paged_append(b.cache, b.K, b.V, b.cu_d, b.lens_d, wide, wide_v, b.table_d, rope=rope, Q=b.Q, Q_out=q)
    y = orc.turn(f64(b.Q).transpose(1, 0, 2), np.concatenate([np.arange(n - m, n) for m, n in zip([3, 17, 0, 1], [40, 17, 3, 64])])[None], [64])
    bound = norm_bound(f64(b.Q).transpose(1, 0, 2), "bf16", y, pairs=[64])
    assert all((np.abs(f64(x).transpose(1, 0, 2) - y) <= bound).all() for x in (out, q))
    written = (wide_v != 0).any(-1).cpu().numpy()
    assert written.sum() == 21 * 3
    for codes, scales, want in ((b.K_pages, b.K_scales, wide), (b.V_pages, b.V_scales, wide_v)):
        got, want = values(codes, scales)[written], f64(want)[written]
        top = np.abs(want).max(-1, keepdims=True)
        assert (np.abs(got - want) <= (2.0 ** -4 + 2.0 ** -8) * np.abs(want) + 2.0 ** -10 / 448 * top * 1.01).all()
