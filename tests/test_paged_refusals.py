"""Calls over a cache of pages that would write over what they read: refused on the host, no kernel is launched here."""
import ctypes

import pytest

import paper_2604_10103_amd as hf

Q, K, V, OUT, TABLES, KP, VP, WS = (i << 24 for i in range(1, 9))   # addresses, never followed
CU, LENS, TABLE, POS = TABLES, TABLES + 4096, TABLES + 8192, TABLES + 12288
N, SEQS, PAGES = 5, 3, 4


def _cache():
    return hf.make_paged(heads=8, heads_kv=2, head_dim=64, dtype="bf16", page_tokens=16, n_pages=10, n_seqs=SEQS, max_pages=PAGES)


def _append(lib, rope=True, **kw):
    a = dict(Q=Q, O=OUT, cu=CU, lens=LENS, table=TABLE, pos=POS, KP=KP, VP=VP, n=N)
    a.update(kw)
    r = ctypes.byref(hf.make_rope_axes([8, 8])) if rope else None
    return lib.hf_paged_append(ctypes.byref(_cache()), r, a["n"], K, None, V, None, a["Q"], None, a["cu"], a["lens"], a["pos"], a["KP"], a["VP"],
                               a["table"], a["O"], None, None)


def _attend(lib, **kw):
    cache = _cache()
    a = dict(O=OUT, lse=OUT + (1 << 20), cu=CU, lens=LENS, table=TABLE, ws=WS, size=hf.hf_paged_workspace_bytes(cache, N))
    a.update(kw)
    return lib.hf_paged_attn_fwd(ctypes.byref(cache), Q, None, N, a["cu"], a["lens"], KP, VP, a["table"], a["O"], None, a["lse"], a["ws"],
                                 a["size"], None)


# bytes of what the device reads
READS = dict(cu=4 * (SEQS + 1), lens=4 * SEQS, table=4 * SEQS * PAGES, pos=4 * 2 * N)
POOL = 10 * 2 * 16 * 64 * 2


@pytest.mark.parametrize("read", ["cu", "lens", "table", "pos"])
@pytest.mark.parametrize("into,size", [(OUT, N * 8 * 64 * 2), (KP, POOL), (VP, POOL)])
def test_append_does_not_write_over_lengths_tables_and_positions(read, into, size):
    lib = hf.load()
    for at in (into, into + size - 4, into - READS[read] + 4):   # its first word, its last one, the read one's last word
        assert _append(lib, **{read: at}) == -2
        assert b"overlaps" in lib.hf_last_error()


@pytest.mark.parametrize("read", ["cu", "lens", "table"])
def test_attention_does_not_write_over_lengths_and_tables(read):
    lib = hf.load()
    need = hf.hf_paged_workspace_bytes(_cache(), N)
    assert need > 0
    for into, size in ((OUT, N * 8 * 64 * 2), (OUT + (1 << 20), 8 * N * 4), (WS, need)):
        for at in (into, into + size - 4, into - READS[read] + 4):
            assert _attend(lib, **{read: at}) == -2
            assert b"overlaps" in lib.hf_last_error()


def _large(n_seqs, heads, heads_kv, head_dim=64, dtype="bf16"):
    return hf.make_paged(heads=heads, heads_kv=heads_kv, head_dim=head_dim, dtype=dtype, page_tokens=64, n_pages=1000, n_seqs=n_seqs, max_pages=8)


@pytest.mark.parametrize("n_seqs,new,heads,heads_kv,head_dim,dtype", [(65535, 33, 256, 256, 64, "bf16"), (65535, 33, 256, 256, 128, "f32"),
                                                                     (65535, 40, 400, 400, 128, "bf16")])
def test_more_workgroups_than_a_launch_has(n_seqs, new, heads, heads_kv, head_dim, dtype):
    """2^32 threads or more: refused by both calls alike, before anything else is looked at."""
    lib, c, n = hf.load(), _large(n_seqs, heads, heads_kv, head_dim, dtype), n_seqs * new
    assert n * heads <= 1 << 30 and (n * heads // 128 + n_seqs * heads_kv) * 256 >= 1 << 32
    with pytest.raises(hf.HFError, match="threads") as e:
        hf.hf_paged_workspace_bytes(c, n)
    assert e.value.code == -2
    assert lib.hf_paged_attn_fwd(ctypes.byref(c), None, None, n, CU, LENS, KP, VP, TABLE, OUT, None, None, None, 0, None) == -2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("n_seqs,n,heads,heads_kv", [(1, 1 << 22, 256, 256), (1, 1 << 24, 64, 1), (65535, 65535, 16384, 16384), (65535, 65535 * 33, 64, 32),
                                                     (1, 0, 65535, 65535)])
def test_large_calls_that_a_launch_can_hold(n_seqs, n, heads, heads_kv, head_dim, dtype):
    hf.hf_paged_workspace_bytes(_large(n_seqs, heads, heads_kv, head_dim, dtype), n)
