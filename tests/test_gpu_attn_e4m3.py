"""Attention over pages in 8 bits against the 64-bit oracle on what the codes stand for, element by element (bounds: tests/e4m3.py)."""
import numpy as np
import pytest
import torch

import paper_2604_10103_amd as hf
from e4m3 import Batch8
from paged import DEV, f64

pytestmark = pytest.mark.gpu

MASKS = {"causal": dict(causal=True), "all": dict(causal=False), "window": dict(causal=True, window=19, n_sink=3),
         "frames": dict(causal=False, window=40, n_sink=8)}
BATCHES = {   # new tokens, lengths
    "one": ([1], [1]), "short": ([1], [118]), "tokens": ([1, 1, 0, 1, 1], [3, 200, 7, 64, 33]), "drafts": ([4, 2, 4, 1], [70, 131, 4, 1]),
    "chunk": ([50], [173]), "prompts": ([33, 1, 70, 0], [33, 90, 201, 5]), "before": ([9, 3], [4, 2]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", list(MASKS))
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("heads,heads_kv,page", [(3, 3, 16), (8, 2, 7), (6, 1, 40)])
def test_attention(dtype, d, mask, batch, heads, heads_kv, page):
    new, lens = BATCHES[batch]
    b = Batch8(new, lens, heads, heads_kv, d, dtype, page, rows_behind=3, seed=d + page, **MASKS[mask])
    O, lse2 = b.attend()
    b.check(O, lse2)
    again, lse_again = b.attend()
    assert torch.equal(O, again) and torch.equal(lse2, lse_again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens,heads,heads_kv,d,page,kw", [
    ([1], [9000], 8, 2, 128, 64, {}), ([4], [5000], 32, 8, 128, 16, {}), ([2] * 3, [4001, 30, 1999], 4, 4, 64, 33, {}),
    ([1] * 40, list(range(1, 4000, 100)), 8, 8, 128, 16, {}), ([1] * 300, [5 + 7 * (i % 40) for i in range(300)], 8, 8, 64, 16, {}),
    ([1] * 70, [1 + i for i in range(70)], 40, 40, 64, 5, {}), ([300], [2100], 4, 1, 128, 64, {}), ([260, 130], [900, 130], 12, 12, 128, 100, {}),
    ([513], [1500], 8, 8, 64, 256, dict(causal=False)), ([700], [1400], 3, 3, 128, 350, dict(causal=False, window=700, n_sink=350)),
    ([1], [20000], 1, 1, 128, 16, dict(window=9000, n_sink=70)), ([1], [4000], 16, 1, 128, 4000, {}), ([1], [4000], 32, 1, 64, 1, {}),
    ([3], [3000], 24, 2, 128, 48, dict(gain=6.0)), ([200], [600], 4, 2, 128, 48, dict(gain=6.0)),
    # 16 and 32 rows by eight wavefronts, four, and one
    ([1] * 90, [7 * i + 1 for i in range(90)], 8, 8, 128, 16, {}), ([6] * 10, [300 * i + 6 for i in range(10)], 8, 2, 128, 64, {}),
    ([6] * 70, [6 + 5 * i for i in range(70)], 32, 8, 64, 16, {}), ([5] * 330, [5 + i % 60 for i in range(330)], 16, 4, 128, 16, {})])
def test_longer(dtype, new, lens, heads, heads_kv, d, page, kw):
    b = Batch8(new, lens, heads, heads_kv, d, dtype, page, seed=len(lens) + d, **kw)
    O, lse2 = b.attend()
    b.check(O, lse2)
    again, _ = b.attend()
    assert torch.equal(O, again)


def _reference(b):
    """The oracle's answer by 64-bit products on the GPU, for many rows."""
    n, d, group = b.n, b.d, b.heads // b.heads_kv
    R, spread = np.full((n, b.heads, d), np.nan), np.full((n, b.heads, d), np.nan)
    L, size, count = np.full((b.heads, n), np.nan), np.zeros((n, b.heads)), np.zeros(n, dtype=int)
    K, V = (c.float().double() * s.double()[..., None] for c, s in ((b.K_pages, b.K_scales), (b.V_pages, b.V_scales)))
    for s in range(len(b.lens)):
        m, length, rows = int(b.cu[s + 1] - b.cu[s]), int(b.lens[s]), slice(int(b.cu[s]), int(b.cu[s + 1]))
        pages = torch.tensor(b.table[s, :-(-length // b.page)], dtype=torch.long, device=DEV)
        p, j = torch.arange(length - m, length, device=DEV)[:, None], torch.arange(length, device=DEV)[None]
        sees = j <= p if b.mask["causal"] else j >= 0
        if b.mask["window"]:
            sees = sees & ((j > p - b.mask["window"]) | (j < b.mask["n_sink"]))
        sees = sees.expand(m, length)
        count[rows] = sees.sum(1).cpu().numpy()
        for h in range(b.heads):
            k, v = (x[pages, h // group].flatten(0, 1)[:length].contiguous() for x in (K, V))
            q = b.Q[rows, h].double()
            logit = (q @ k.T.contiguous() / d ** 0.5).masked_fill(~sees, -float("inf"))
            w = torch.softmax(logit, -1)
            R[rows, h], spread[rows, h] = f64(w @ v), f64(w @ v.abs())
            L[h, rows] = f64(torch.logsumexp(logit, -1)) / np.log(2.0)
            size[rows, h] = f64((q.abs() @ k.abs().T.contiguous() / d ** 0.5 * sees).amax(-1))
    return R, L, spread, size, count


@pytest.mark.parametrize("mask", [dict(causal=True), dict(causal=False, window=300, n_sink=70)])
@pytest.mark.parametrize("new,lens,heads,heads_kv,page", [([600], [703], 64, 64, 50), ([513, 700], [513, 1500], 48, 24, 256), ([300], [2000], 64, 8, 16)])
def test_256_rows_a_workgroup(mask, new, lens, heads, heads_kv, page):
    b = Batch8(new, lens, heads, heads_kv, 128, "bf16", page, rows_behind=2, seed=page, **mask)
    O, lse2 = b.attend()
    b.check(O, lse2, _reference(b))
    free = np.ones((b.n_pages, page), dtype=bool)              # what lies behind the sequences, in their pages and in others
    for s, n in enumerate(lens):
        for j in range(n):
            free[b.table[s, j // page], j % page] = False
    free = torch.tensor(free, device=DEV)[:, None].expand(b.K_scales.shape)
    for codes, scales, x in ((b.K_pages, b.K_scales, float("inf")), (b.V_pages, b.V_scales, float("nan"))):
        codes.view(torch.uint8)[free] = 0x7f
        scales[free] = x
    again, lse_again = b.attend()
    assert torch.equal(O, again) and torch.equal(lse2, lse_again)


def test_the_reference_is_the_oracle():
    b = Batch8([5, 30], [90, 61], 6, 2, 64, "f32", 16, seed=1, causal=True, window=20, n_sink=3)
    for x, y in zip(_reference(b), b.oracle()):
        np.testing.assert_allclose(x, y, rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens", [([1, 2], [90, 75]), ([40, 3], [90, 75])])
def test_what_a_token_does_not_see_is_nothing_to_it(dtype, new, lens):
    """NaN codes, scales that are not finite and entries that are no page, everywhere where a token does not look."""
    for kw in (dict(causal=True, window=21, n_sink=5), dict(causal=True)):
        b = Batch8(new, lens, 6, 2, 128, dtype, 16, rows_behind=2, seed=8, extra_entries=2, **kw)
        O, lse2 = b.attend()
        held = np.zeros(b.K_scales.shape[:1] + (16,), dtype=bool)
        for s, n in enumerate(lens):
            first = n - new[s] - 20 if "window" in kw else 0   # the first new token's window
            for j in range(n):
                if j >= first or j < 5:
                    held[b.table[s, j // 16], j % 16] = True
        free = torch.tensor(~held, device=DEV)[:, None].expand(b.K_scales.shape)
        for codes, scales, s in ((b.K_pages, b.K_scales, float("nan")), (b.V_pages, b.V_scales, float("inf"))):
            raw = codes.view(torch.uint8)
            raw[free] = torch.tensor([0x7f, 0xff] * 64, dtype=torch.uint8, device=DEV)
            scales[free] = s
        again, lse_again = b.attend()
        assert torch.equal(O, again) and torch.equal(lse2, lse_again)
        b.table[:, -2:] = -5
        b.to_gpu()
        again, _ = b.attend()
        assert torch.equal(O, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens", [([6], [200]), ([60], [200])])
@pytest.mark.parametrize("heads", [2, 6])
def test_a_nan_reaches_who_sees_it(dtype, new, lens, heads):
    """A NaN code of a value: that feature of the rows that see it; of a key, or a scale: the whole rows.  All others keep their bits."""
    b = Batch8(new, lens, heads, 2, 64, dtype, 16, seed=3)
    O, _ = b.attend()
    m = new[0]
    for place in (lens[0] - m // 2, 3):
        sees = np.arange(lens[0] - m, lens[0]) >= place
        page, at = int(b.table[0, place // 16]), place % 16
        for what in ("v", "k", "ks", "vs"):
            codes, scales = (b.K_pages, b.K_scales) if what[0] == "k" else (b.V_pages, b.V_scales)
            raw = codes.view(torch.uint8)
            kept = raw[page, 1, at].clone(), scales[page, 1, at].clone()
            if what in "kv":
                raw[page, 1, at, 37] = 0xff if what == "k" else 0x7f
            else:
                scales[page, 1, at] = float("nan")
            got, _ = b.attend()
            raw[page, 1, at], scales[page, 1, at] = kept
            bad = torch.zeros(b.n, heads, 64, dtype=torch.bool)
            bad[torch.tensor(sees), heads // 2:, (slice(37, 38) if what == "v" else slice(None))] = True
            nan = torch.isnan(got).cpu()
            assert torch.equal(nan, bad), (what, place)
            assert torch.equal(got.cpu()[~bad], O.cpu()[~bad])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[2, 1, 1], [40, 1, 30]])
def test_rows_that_see_nothing(dtype, new):
    """No page where all of a sequence's keys would be; a sequence without length; lengths below the new tokens."""
    b = Batch8(new, [max(new), 50, 0], 4, 2, 64, dtype, 16, rows_behind=2, seed=5)
    b.table[1] = -1
    b.to_gpu()
    O, lse2 = b.attend()
    b.check(O, lse2)
    rows = slice(int(b.cu[1]), int(b.cu[3]))
    assert (O[rows] == 0).all() and torch.isposinf(lse2[:, rows]).all()


@pytest.mark.parametrize("new", [[1, 3], [64, 20]])
def test_a_missing_page_in_the_middle(new):
    for dtype in ("bf16", "f32"):
        b = Batch8(new, [300, 210], 8, 2, 128, dtype, 16, seed=6)
        b.table[0, 3], b.table[1, 0], b.table[1, 7] = -1, b.n_pages, 2 ** 31 - 1
        b.to_gpu()
        b.check(*b.attend())


def test_scale_strides_and_no_lse():
    b = Batch8([2, 30], [77, 90], 8, 4, 64, "bf16", 16, seed=7, scale=0.3)
    O, _ = b.attend(lse=False)
    b.check(O, None)
    wide = torch.full((b.n, 3, 8, 64), 7.0, dtype=b.t, device=DEV)
    hf.hf_paged_attn_e4m3_fwd(b.cache, b.Q, b.cu_d, b.lens_d, b.K_pages, b.V_pages, b.K_scales, b.V_scales, b.table_d, wide[:, 1], b.workspace())
    assert torch.equal(wide[:, 1], O) and (wide[:, ::2] == 7).all()


def test_extreme_scales():
    """Rows of very different sizes: a key's score and a value's share are as large as its scale makes them."""
    for dtype in ("bf16", "f32"):
        for new in ([2], [50]):
            b = Batch8(new, [150], 4, 2, 64, dtype, 16, seed=9, spread=4.0)
            b.K_scales.mul_(0.02)
            b.check(*b.attend())


def test_two_graphs_and_streams_follow_lengths():
    """One workspace for two graphs that do not overlap, lengths and tables changed between replays."""
    bs = [Batch8([1, 1, 1], [900, 1500, 3], 8, 2, 128, "bf16", 16, seed=1), Batch8([40, 1, 9], [400, 700, 30], 8, 2, 128, "bf16", 16, seed=2)]
    ws = torch.zeros(max(hf.hf_paged_e4m3_workspace_bytes(b.cache, b.n) for b in bs), dtype=torch.uint8, device=DEV)
    outs, graphs = [], []
    for b in bs:
        O = torch.empty(b.n, 8, 128, dtype=b.t, device=DEV)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b.attend(lse=False, O=O, workspace=ws)
        outs.append(O)
        graphs.append(graph)
    for k in range(4):
        for b, O, graph in zip(bs, outs, graphs):
            b.lens[:] = np.maximum(b.lens - 3 * k, b.cu[1:] - b.cu[:-1])
            b.lens_d.copy_(torch.tensor(b.lens, dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            want, _ = b.attend(lse=False)
            assert torch.equal(O, want)
            if k in (0, 3):
                b.check(O, None)


def test_a_layer_of_serving():
    """Append and attention as they are used: prompts, then single tokens, in bf16, against the oracle on the cache's contents; the same in
    a captured step."""
    from e4m3 import rope_of
    heads, heads_kv, d, P, S, steps = 8, 2, 128, 16, 3, 4
    prompts = [37, 5, 80]
    g = torch.Generator().manual_seed(12)
    pages = sum(-(-(p + steps) // P) for p in prompts)
    table = np.full((S, 6), -1, dtype=np.int32)
    at = 0
    for s, p in enumerate(prompts):
        k = -(-(p + steps) // P)
        table[s, :k] = np.arange(at, at + k)[::-1]
        at += k
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    codes = [torch.zeros(pages, heads_kv, P, d, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in "kv"]
    scales = [torch.zeros(pages, heads_kv, P, device=DEV) for _ in "kv"]
    cache = hf.make_paged(heads, heads_kv, d, "bf16", P, pages, S, 6)
    norm, rope = hf.make_head_norm(), rope_of([64])
    scaling = hf.make_rope_scaling(2.0, 64.0, slow=1.0, fast=8.0)
    w = [torch.randn(d, generator=g).to(DEV) for _ in "kq"]
    tab, lens = ints(table), ints(prompts)

    def layer(x, cu, ws):
        Q, K, V = x[:, :heads], x[:, heads:heads + heads_kv], x[:, heads + heads_kv:]
        q = torch.empty(len(x), heads, d, dtype=torch.bfloat16, device=DEV)
        hf.hf_paged_append_e4m3(cache, K, V, cu, lens, *codes, *scales, tab, norm=norm, k_weight=w[0], q_weight=w[1], rope=rope,
                                scaling=scaling, Q=Q, Q_out=q)
        O = torch.empty_like(q)
        hf.hf_paged_attn_e4m3_fwd(cache, q, cu, lens, *codes, *scales, tab, O, ws)
        return q, O

    def check(q, O, new):
        b = Batch8.__new__(Batch8)
        b.dtype, b.d, b.scale, b.mask = "bf16", d, 0.0, dict(causal=True, window=0, n_sink=0)
        b.Q, (b.K_pages, b.V_pages), (b.K_scales, b.V_scales), b.table = q, codes, scales, table
        b.cu, b.lens = np.concatenate([[0], np.cumsum(new)]), lens.cpu().numpy()
        b.check(O, None)

    size = max(hf.hf_paged_e4m3_workspace_bytes(cache, n) for n in (sum(prompts), S))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    x = torch.randn(sum(prompts), heads + 2 * heads_kv, d, generator=g).to(torch.bfloat16).to(DEV)
    check(*layer(x, ints(np.concatenate([[0], np.cumsum(prompts)])), ws), prompts)
    x, cu = torch.zeros(S, heads + 2 * heads_kv, d, dtype=torch.bfloat16, device=DEV), ints(np.arange(S + 1))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        q, O = layer(x, cu, ws)
    for _ in range(steps):
        lens += 1
        x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        check(q, O, [1] * S)
    assert f64(scales[0]).min() >= 0


def test_two_calls_at_once():
    """Two streams, a workspace each; and a stream other than the tensors' own."""
    bs = [Batch8([1] * 4, [3000, 50, 900, 2100], 8, 2, 128, "bf16", 16, seed=21), Batch8([60, 2], [900, 700], 8, 2, 128, "bf16", 16, seed=22)]
    want = [b.attend(lse=False)[0] for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for b, stream in zip(bs, streams):
            with torch.cuda.stream(stream):
                got.append(b.attend(lse=False)[0])
    torch.cuda.synchronize()
    for k, O in enumerate(got):
        assert torch.equal(O, want[k % 2])
