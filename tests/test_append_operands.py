"""Both appends: queries that are written lie between the new keys' and values' rows, or apart from them, but over none of their elements.  The
refusals are the host's: no kernel is launched but in the tests that are marked for a GPU."""
import ctypes
import random

import pytest
import torch

import paper_2604_10103_amd as hf
from paged import DEV

BASE, FAR = 1 << 30, [i << 40 for i in range(1, 9)]      # addresses, never followed
HEADS, KV, D, N = 4, 2, 64, 5
ROW = 2 * D                                               # bytes of a row in bf16


@pytest.fixture(scope="module")
def lib():
    return hf.load()


def _strides(s):
    return (ctypes.c_int64 * 2)(*[x // 2 for x in s])


def _call(lib, wide, q_out, qs, k, ks, v, vs, pages=FAR[0]):
    """The refusal of an append with these addresses and (row, head) strides in bytes; it has one: the pages lie over the queries, which is
    found last, where `pages` does."""
    cache = ctypes.byref(hf.make_paged(HEADS, KV, D, "bf16", 16, 10, 3, 4))
    q, cu, lens, vp, kscales, vscales, table = FAR[1:8]
    args = [N, k, _strides(ks), v, _strides(vs), q, None]
    if wide:
        rc = lib.hf_paged_append(cache, None, *args, cu, lens, None, pages, vp, table, q_out, _strides(qs), None)
    else:
        rc = lib.hf_paged_append_e4m3(cache, None, None, None, *args, None, None, cu, lens, None, pages, vp, kscales, vscales, table, q_out,
                                      _strides(qs), None)
    assert rc == -2
    return lib.hf_last_error().decode()


def _joint(order):
    """Offsets and (row, head) strides of Q_out, K_new and V_new in one buffer, the queries' last element at its end."""
    if order == "rows":            # [token, keys | values | queries, d]
        s = ((HEADS + 2 * KV) * ROW, ROW)
        return (2 * KV * ROW, s), (0, s), (KV * ROW, s)
    if order == "heads":           # [token, head, key | value | query, d], two query heads for each key head
        s, q = (KV * 4 * ROW, 4 * ROW), (KV * 4 * ROW, 2 * ROW)
        return (ROW, q), (0, s), (2 * ROW, s)
    if order == "head first":      # [head, key | value | query, token, d], the queries' heads twice as close as the keys'
        s, q = (ROW, 4 * N * ROW), (ROW, 2 * N * ROW)
        return (N * ROW, q), (0, s), (2 * N * ROW, s)
    if order == "pieces":          # 16 bytes between any two rows
        s = ((HEADS + 2 * KV) * (ROW + 16), ROW + 16)
        return (2 * KV * (ROW + 16), s), (0, s), (KV * (ROW + 16), s)
    if order == "every second":    # keys and values of another projection lie two tokens' rows apart, between the queries'
        s = ((HEADS + KV) * ROW, ROW)
        return (KV * ROW, s), (0, (2 * s[0], ROW)), (s[0], (2 * s[0], ROW))
    s = (0, ROW)                   # one key, one value for all tokens
    return (2 * KV * ROW, (HEADS * ROW, ROW)), (0, s), (KV * ROW, s)


ORDERS = ["rows", "heads", "head first", "pieces", "every second", "one for all"]


def _bytes_of(at, strides, heads):
    return {at + i * strides[0] + h * strides[1] + b for i in range(N) for h in range(heads) for b in range(0, ROW, 16)}


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("order", ORDERS)
def test_interleaved_operands_are_no_overlap(lib, wide, order):
    (q, qs), (k, ks), (v, vs) = _joint(order)
    assert not _bytes_of(q, qs, HEADS) & (_bytes_of(k, ks, KV) | _bytes_of(v, vs, KV))
    # pages behind all that the keys and values span, over the queries' last row or, where those reach further, over all: found after the rest
    end = max(_bytes_of(q, qs, HEADS)) - 16
    if end > max(_bytes_of(k, ks, KV) | _bytes_of(v, vs, KV)):
        message = _call(lib, wide, BASE + q, qs, BASE + k, ks, BASE + v, vs, pages=BASE + end)
        assert message in ("Q_out overlaps K_pages", "Q_out overlaps the pages")
    # one row further the queries lie over keys or values, one of which is named
    for by in (16, -16, ROW - 16):
        moved = q + by
        if moved >= 0 and _bytes_of(moved, qs, HEADS) & (_bytes_of(k, ks, KV) | _bytes_of(v, vs, KV)):
            message = _call(lib, wide, BASE + moved, qs, BASE + k, ks, BASE + v, vs)
            assert message in ("Q_out overlaps K_new", "Q_out overlaps V_new")


@pytest.mark.parametrize("wide", [False, True])
def test_queries_over_keys_or_values(lib, wide):
    (q, qs), (k, ks), (v, vs) = _joint("rows")
    far = FAR[0] >> 1
    assert _call(lib, wide, BASE, qs, BASE, ks, far, vs) == "Q_out overlaps K_new"
    assert _call(lib, wide, BASE, qs, far, ks, BASE + ROW, vs) == "Q_out overlaps V_new"
    packed = (HEADS * ROW, ROW)
    assert _call(lib, wide, BASE, packed, BASE + N * HEADS * ROW - ROW, (KV * ROW, ROW), far, vs) == "Q_out overlaps K_new"


@pytest.mark.parametrize("wide", [False, True])
def test_no_shared_element_is_accepted(lib, wide):
    """Random strides and places, against the sets of what they cover."""
    rng, shared = random.Random(5), 0
    far = FAR[0] >> 1
    for _ in range(1500):
        head = rng.choice([ROW, ROW + 16, 2 * ROW, 3 * ROW])
        qs = (HEADS * head + 16 * rng.randrange(0, 30), head)
        ks = rng.choice([qs, (2 * qs[0], head), (qs[0], 2 * head), (0, head), (16 * rng.randrange(0, 80), 16 * rng.randrange(0, 20))])
        k = 16 * rng.randrange(0, 300)
        q = 16 * rng.randrange(0, 300)
        if _bytes_of(q, qs, HEADS) & _bytes_of(k, ks, KV):
            shared += 1
            assert _call(lib, wide, BASE + q, qs, BASE + k, ks, far, (KV * ROW, ROW)) == "Q_out overlaps K_new"
    assert shared > 300


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("order", ORDERS)
def test_interleaved_operands(wide, order):
    """The same keys, values and queries in one buffer and apart: the same pages and queries, in place and into rows between the keys'."""
    places = _joint(order)
    size = max(max(_bytes_of(at, s, h)) for (at, s), h in zip(places, (HEADS, KV, KV))) + 16
    g = torch.Generator().manual_seed(3)
    buffer = torch.randn(size // 2, generator=g).to(torch.bfloat16).to(DEV)
    take = lambda b: [torch.as_strided(b, (N, h, D), (s[0] // 2, s[1] // 2, 1), at // 2) for (at, s), h in zip(places, (HEADS, KV, KV))]  # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    rope = hf.make_rope_axes([16])

    def append(Q, K, V, out):
        table = ints([1, 0])
        cache = hf.make_paged(HEADS, KV, D, "bf16", 4, 2, 1, 2)
        shape = (2, KV, 4, D)
        if wide:
            pages = [torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
            hf.hf_paged_append(cache, K, V, ints(0, N), ints(N), *pages, table, rope=rope, Q=Q, Q_out=out)
            return pages
        pages = [torch.zeros(shape, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in "kv"]
        scales = [torch.zeros(shape[:3], device=DEV) for _ in "kv"]
        hf.hf_paged_append_e4m3(cache, K, V, ints(0, N), ints(N), *pages, *scales, table, norm=hf.make_head_norm(), rope=rope, Q=Q, Q_out=out)
        return [p.view(torch.uint8) for p in pages] + scales

    Q, K, V = [x.clone() for x in take(buffer)]
    want_q = torch.empty(N, HEADS, D, dtype=torch.bfloat16, device=DEV)
    want = append(Q.contiguous(), K.contiguous(), V.contiguous(), want_q)
    for in_place in (True, False):
        b = buffer.clone()
        q, k, v = take(b)
        got = append(q if in_place else Q.contiguous(), k, v, q)
        assert torch.equal(q, want_q) and torch.equal(k, K) and torch.equal(v, V)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
