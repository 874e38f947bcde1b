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
