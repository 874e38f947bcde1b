"""Norms with rotation and the pages in 8 bits: structure layouts, refusals and host-only sizes.  No kernel is launched here."""
import ctypes

import pytest
import torch

import paper_2604_10103_amd as hf

X, Y, DX, W, DW, POS, WS = (i << 24 for i in range(1, 8))                        # addresses, never followed
K, V, Q, O, CU, LENS, TABLE, KP, VP, KS, VS = (i << 24 for i in range(9, 20))
N, SEQS, PAGES = 5, 3, 4


@pytest.fixture(scope="module")
def lib():
    return hf.load()


def _ref(s):
    return None if s is None else ctypes.byref(s)


def _fwd(lib, norm=hf.make_head_norm(), rope=hf.make_rope_axes([8, 8]), scaling=None, **kw):
    a = dict(dtype=0, d=64, B=2, H=4, n=N, x=X, xs=None, w=W, pos=POS, per_batch=0, y=Y, ys=None)
    a.update(kw)
    return lib.hf_norm_rope_fwd(_ref(norm), _ref(rope), _ref(scaling), a["dtype"], a["d"], a["B"], a["H"], a["n"], a["x"], a["xs"], a["w"], a["pos"],
                                a["per_batch"], a["y"], a["ys"], None)


def _bwd(lib, norm=hf.make_head_norm(), rope=hf.make_rope_axes([8, 8]), scaling=None, **kw):
    a = dict(dtype=0, d=64, B=2, H=4, n=N, x=X, xs=None, w=W, pos=POS, dy=Y, dys=None, dx=DX, dxs=None, dw=DW, ws=WS)
    a.update(kw)
    size = a.get("size", hf.hf_norm_rope_bwd_workspace_bytes(hf.make_head_norm(), 64, 2, 4, N))
    return lib.hf_norm_rope_bwd(_ref(norm), _ref(rope), _ref(scaling), a["dtype"], a["d"], a["B"], a["H"], a["n"], a["x"], a["xs"], a["w"], a["pos"], 0,
                                a["dy"], a["dys"], a["dx"], a["dxs"], a["dw"], a["ws"], size, None)


def _cache(**kw):
    a = dict(heads=8, heads_kv=2, head_dim=64, dtype="bf16", page_tokens=16, n_pages=10, n_seqs=SEQS, max_pages=PAGES)
    a.update(kw)
    return hf.make_paged(**a)


def _append(lib, norm=hf.make_head_norm(), rope=hf.make_rope_axes([8, 8]), scaling=None, cache=None, **kw):
    a = dict(n=N, k=K, ks=None, v=V, vs=None, q=Q, qs=None, kw=W, qw=DW, cu=CU, lens=LENS, pos=POS, KP=KP, VP=VP, KS=KS, VS=VS, table=TABLE, o=O,
             os=None)
    a.update(kw)
    return lib.hf_paged_append_e4m3(_ref(cache or _cache()), _ref(norm), _ref(rope), _ref(scaling), a["n"], a["k"], a["ks"], a["v"], a["vs"], a["q"],
                                    a["qs"], a["kw"], a["qw"], a["cu"], a["lens"], a["pos"], a["KP"], a["VP"], a["KS"], a["VS"], a["table"],
                                    a["o"], a["os"], None)


def _attend(lib, cache=None, **kw):
    cache = cache or _cache()
    a = dict(q=Q, qs=None, n=N, cu=CU, lens=LENS, KP=KP, VP=VP, KS=KS, VS=VS, table=TABLE, o=O, os=None, lse=DW, ws=WS)
    a.update(kw)
    size = a.get("size", hf.hf_paged_e4m3_workspace_bytes(_cache(), N))
    return lib.hf_paged_attn_e4m3_fwd(_ref(cache), a["q"], a["qs"], a["n"], a["cu"], a["lens"], a["KP"], a["VP"], a["KS"], a["VS"], a["table"], a["o"],
                                      a["os"], a["lse"], a["ws"], size, None)


def _strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


def test_structure_layouts():
    assert ctypes.sizeof(hf.hf_head_norm) == 8 and ctypes.sizeof(hf.hf_rope_scaling) == 40
    assert hf.hf_rope_scaling.amplitude.offset == 32 and hf.hf_rope_scaling.axes.offset == 36
    assert hf.make_rope_scaling(2.0, 10.0, axes=[0, 2, 2]).axes == 5


@pytest.mark.parametrize("call", [_fwd, _bwd, _append])
@pytest.mark.parametrize("kw,code", [
    (dict(norm=hf.make_head_norm(eps=-1.0)), -2), (dict(norm=hf.make_head_norm(eps=float("nan"))), -2), (dict(rope=hf.make_rope_axes([33])), -2),
    (dict(scaling=hf.make_rope_scaling(0.5, 10)), -2), (dict(scaling=hf.make_rope_scaling(float("inf"), 10)), -2),
    (dict(scaling=hf.make_rope_scaling(2, 0)), -2), (dict(scaling=hf.make_rope_scaling(2, float("nan"))), -2),
    (dict(scaling=hf.make_rope_scaling(2, 10, slow=4, fast=4)), -2), (dict(scaling=hf.make_rope_scaling(2, 10, slow=-1)), -2),
    (dict(scaling=hf.make_rope_scaling(2, 10, fast=float("inf"))), -2), (dict(scaling=hf.make_rope_scaling(2, 10, amplitude=0)), -2),
    (dict(scaling=hf.make_rope_scaling(2, 10, amplitude=float("nan"))), -2), (dict(scaling=hf.make_rope_scaling(2, 10, axes=[2])), -2),
    (dict(scaling=hf.make_rope_scaling(2, 10), rope=None), -1), (dict(n=-1), -2), (dict(n=(1 << 24) + 1), -2)])
def test_bad_norms_turns_and_scalings(lib, call, kw, code):
    assert call(lib, **kw) == code


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("kw,code", [
    (dict(d=96), -2), (dict(dtype=3), -3), (dict(B=0), -2), (dict(H=0), -2), (dict(H=65536), -2), (dict(x=None), -1), (dict(x=X + 8), -4),
    (dict(norm=None, rope=None, w=None, dw=None), -1), (dict(norm=None, dw=None), -1), (dict(pos=None), -1), (dict(w=W + 2), -4),
    (dict(xs=_strides(1280, 320, -64)), -2), (dict(xs=_strides(2560, 640, 60)), -4), (dict(w=Y), -2), (dict(pos=Y + 16), -2)])
def test_norm_arguments(lib, call, kw, code):
    if call is _bwd:   # what it writes is dX
        kw = {k: v + DX - Y if k in ("w", "pos") and v and v >= Y and v < Y + 64 else v for k, v in kw.items()}
    assert call(lib, **kw) == code


def test_outputs_of_norms(lib):
    assert _fwd(lib, y=None) == -1 and _fwd(lib, y=Y + 4) == -4
    assert _fwd(lib, y=X + 64) == -2 and b"overlaps" in lib.hf_last_error()
    assert _fwd(lib, ys=_strides(0, 320, 64)) == -2                              # rows over each other
    assert _bwd(lib, dx=X + 64) == -2 and _bwd(lib, dx=Y + 64) == -2
    assert _bwd(lib, norm=None, w=None) == -1                                    # dweight without norm
    assert _bwd(lib, ws=None) == -5 and _bwd(lib, size=0) == -5 and _bwd(lib, ws=WS + 16) == -4
    for kw in (dict(dw=X), dict(dw=Y + 16), dict(dw=DX), dict(dw=W), dict(dw=POS), dict(ws=X), dict(ws=Y), dict(ws=DX), dict(ws=DW), dict(ws=POS)):
        assert _bwd(lib, **kw) == -2 and b"overlaps" in lib.hf_last_error(), kw
    assert hf.hf_norm_rope_bwd_workspace_bytes(hf.make_head_norm(), 128, 1, 1, 0) == 0
    with pytest.raises(hf.HFError):
        hf.hf_norm_rope_bwd_workspace_bytes(hf.make_head_norm(), 96, 1, 1, 1)
    assert lib.hf_norm_rope_bwd_workspace_bytes(None, 64, 1, 1, 1, ctypes.byref(ctypes.c_size_t())) == -1
    assert _fwd(lib, n=0, x=None, y=None, pos=None) == 0 and _bwd(lib, n=0, x=None, dy=None, dx=None, pos=None, dw=None, ws=None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1), (dict(o=None), -1), (dict(KP=None), -1), (dict(VS=None), -1), (dict(KS=KS + 2), -4),
    (dict(KP=KP + 8), -4), (dict(kw=W + 1), -4), (dict(norm=None), -1), (dict(cu=None), -1), (dict(table=None), -1),
    (dict(cache=_cache(n_pages=1 << 30)), -2), (dict(ks=_strides(130, 64)), -4)])
def test_append_arguments(lib, kw, code):
    assert _append(lib, **kw) == code


POOL, SCALES = 10 * 2 * 16 * 64, 10 * 2 * 16 * 4
WRITES = dict(KP=POOL, VP=POOL, KS=SCALES, VS=SCALES)


@pytest.mark.parametrize("written", list(WRITES))
@pytest.mark.parametrize("read", ["k", "v", "q", "kw", "qw", "cu", "lens", "pos", "table", "o", "KP", "VP", "KS", "VS"])
def test_append_writes_over_nothing(lib, written, read):
    if written == read:
        return
    at = {"KP": KP, "VP": VP, "KS": KS, "VS": VS}[written]
    for where in (at, at + (WRITES[written] - 1) // 16 * 16):
        assert _append(lib, **{read: where}) == -2 and b"overlaps" in lib.hf_last_error()


@pytest.mark.parametrize("read", ["kw", "qw", "cu", "lens", "pos", "table"])
def test_rotated_queries_lie_over_no_argument(lib, read):
    assert _append(lib, **{read: O + N * 8 * 64 * 2 - 4}) == -2 and b"Q_out" in lib.hf_last_error()
    assert _append(lib, n=0, **{read: O}) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), -1), (dict(o=None), -1), (dict(KP=None), -1), (dict(VP=VP + 4), -4), (dict(KS=None), -1), (dict(VS=VS + 2), -4),
    (dict(lse=DW + 2), -4), (dict(ws=None), -5), (dict(size=100), -5), (dict(ws=WS + 64), -4), (dict(n=-1), -2), (dict(n=1 << 25), -2),
    (dict(cache=_cache(head_dim=32)), -2), (dict(cache=_cache(heads_kv=3)), -2), (dict(cache=_cache(window=-1)), -2)])
def test_attention_arguments(lib, kw, code):
    assert _attend(lib, **kw) == code


@pytest.mark.parametrize("read", ["q", "cu", "lens", "table", "KP", "VP", "KS", "VS"])
def test_attention_writes_over_nothing(lib, read):
    for at, size in ((O, N * 8 * 64 * 2), (DW, 8 * N * 4), (WS, hf.hf_paged_e4m3_workspace_bytes(_cache(), N))):
        for where in (at, at + (size - 1) // 16 * 16):
            assert _attend(lib, **{read: where}) == -2 and b"overlaps" in lib.hf_last_error()
    assert _attend(lib, lse=O) == -2 and _attend(lib, ws=O) == -2 and _attend(lib, ws=DW) == -2


def test_workspace_sizes(lib):
    sizes = [hf.hf_paged_e4m3_workspace_bytes(_cache(n_seqs=s), n) for s, n in ((1, 0), (1, 1), (64, 4096))]
    assert sizes[0] == 0 and sizes == sorted(sizes)
    with pytest.raises(hf.HFError, match="threads"):
        hf.hf_paged_e4m3_workspace_bytes(_cache(n_seqs=65535, heads=400, heads_kv=400, head_dim=128), 65535 * 40)
    hf.hf_paged_e4m3_workspace_bytes(_cache(n_seqs=65535, heads=16384, heads_kv=16384), 65535)


def test_binding_takes_gpu_tensors_of_its_structures_only(lib):
    x = torch.zeros(2, 4, 5, 64)
    with pytest.raises(TypeError):
        hf.hf_norm_rope_fwd(x, x, norm=hf.make_head_norm())
    with pytest.raises(TypeError):
        hf.hf_norm_rope_bwd(x, x, x, norm=1)
    with pytest.raises(TypeError):
        hf.hf_paged_append_e4m3(_cache(), x[0], x[0], x, x, x, x, x, x, x)
    with pytest.raises(TypeError):
        hf.hf_paged_attn_e4m3_fwd(hf.make_rope_axes([8]), x[0], x, x, x, x, x, x, x, x)
