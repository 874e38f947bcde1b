"""Refusals of the rotation by positions and of the cache of pages, on the host: no kernel is launched here."""
import ctypes

import pytest
import torch

import paper_2604_10103_amd as hf

A, B, C, D, E, F = (i << 24 for i in range(1, 7))   # addresses, never followed


@pytest.fixture(scope="module")
def lib():
    return hf.load()


def _cache(**kw):
    base = dict(heads=8, heads_kv=2, head_dim=64, dtype="bf16", page_tokens=16, n_pages=10, n_seqs=3, max_pages=4)
    base.update(kw)
    return hf.make_paged(**base)


def _strides(*v):
    return (ctypes.c_int64 * len(v))(*v)


def test_structure_layouts():
    assert ctypes.sizeof(hf.hf_paged) == 12 * 4 and hf.hf_paged.softmax_scale.offset == 44
    assert ctypes.sizeof(hf.hf_rope_axes) == 40 and hf.hf_rope_axes.pairs.offset == 12 and hf.hf_rope_axes.spectrum.offset == 32


@pytest.mark.parametrize("kw,code", [
    (dict(heads=0), -2), (dict(heads_kv=0), -2), (dict(heads_kv=3), -2), (dict(heads=65536), -2), (dict(head_dim=96), -2), (dict(dtype=5), -3),
    (dict(page_tokens=0), -2), (dict(page_tokens=65537), -2), (dict(n_pages=0), -2), (dict(n_seqs=0), -2), (dict(n_seqs=65536), -2),
    (dict(max_pages=0), -2), (dict(max_pages=1 << 27), -2), (dict(window=-1), -2), (dict(n_sink=-1), -2), (dict(softmax_scale=-1.0), -2),
    (dict(softmax_scale=float("nan")), -2), (dict(softmax_scale=float("inf")), -2)])
def test_bad_caches_are_refused(lib, kw, code):
    with pytest.raises(hf.HFError) as e:
        hf.hf_paged_workspace_bytes(_cache(**kw), 3)
    assert e.value.code == code


@pytest.mark.parametrize("n", [-1, (1 << 24) + 1])
def test_bad_numbers_of_rows_are_refused(lib, n):
    c = ctypes.byref(_cache())
    with pytest.raises(hf.HFError) as e:
        hf.hf_paged_workspace_bytes(_cache(), n)
    assert e.value.code == -2
    assert lib.hf_paged_attn_fwd(c, A, None, n, B, C, D, E, F, A + (1 << 20), None, None, None, 0, None) == -2
    assert lib.hf_paged_append(c, None, n, A, None, B, None, None, None, C, D, None, E, F, A, None, None, None) == -2
    r = ctypes.byref(hf.make_rope_axes([8]))
    assert lib.hf_rope_axes_apply(r, 0, 64, 1, 1, n, A, None, B, 0, C, None, 0, None) == -2


def test_workspace_grows_with_rows_and_no_length_is_needed(lib):
    sizes = [hf.hf_paged_workspace_bytes(_cache(n_seqs=s), n) for s, n in ((1, 0), (1, 1), (64, 64), (64, 4096))]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("kw,code", [
    (dict(pairs=[]), -2), (dict(pairs=[0]), -2), (dict(pairs=[16, -1]), -2), (dict(pairs=[33]), -2), (dict(pairs=[16, 17]), -2),
    (dict(pairs=[2147483647, 2147483647]), -2), (dict(pairs=[8], theta=0.5), -2), (dict(pairs=[8], theta=float("nan")), -2),
    (dict(pairs=[8], theta=float("inf")), -2), (dict(pairs=[8], layout=2), -3), (dict(pairs=[8], spectrum=-1), -3)])
def test_bad_rotations_are_refused(lib, kw, code):
    r = ctypes.byref(hf.make_rope_axes(**kw))
    assert lib.hf_rope_axes_apply(r, 0, 64, 1, 1, 4, A, None, B, 0, C, None, 0, None) == code
    assert lib.hf_paged_append(ctypes.byref(_cache()), r, 4, A, None, B, None, None, None, C, D, None, E, F, A + 4096, None, None, None) == code


def test_more_axes_than_there_are(lib):
    with pytest.raises(ValueError):
        hf.make_rope_axes([1] * 5)


def test_rotation_arguments(lib):
    r = ctypes.byref(hf.make_rope_axes([8]))
    call = lambda rope=r, dtype=0, d=64, batch=1, heads=2, n=4, X=A, xs=None, pos=B, Y=C, ys=None: lib.hf_rope_axes_apply(  # noqa: E731
        rope, dtype, d, batch, heads, n, X, xs, pos, 0, Y, ys, 0, None)
    assert call(rope=None) == -1 and call(X=None) == -1 and call(pos=None) == -1 and call(Y=None) == -1
    assert call(dtype=2) == -3 and call(d=80) == -2 and call(batch=0) == -2 and call(heads=0) == -2 and call(batch=65536) == -2
    assert call(X=A + 8) == -4 and call(Y=C + 2) == -4 and call(pos=B + 2) == -4
    assert call(xs=_strides(512, 256, 60)) == -4                      # 120 bytes between tokens
    assert call(xs=_strides(512, 256, -64)) == -2
    assert call(ys=_strides(512, 0, 64)) == -2                         # heads on top of each other
    assert call(ys=_strides(512, 64, 64)) == -2
    assert call(ys=_strides(512, 64, 120)) == -2                       # a token spans two heads: 128
    assert call(Y=A + 64) == -2                                        # into X, not X
    assert call(Y=A, ys=_strides(0, 64, 128)) == -2                    # X in another order
    assert call(Y=B - 64) == -2                                        # over the positions


def test_append_arguments(lib):
    c, r = ctypes.byref(_cache()), ctypes.byref(hf.make_rope_axes([8]))
    big = 10 * 2 * 16 * 64 * 2
    base = dict(cache=c, rope=r, n=5, K=A, ks=None, V=B, vs=None, Q=None, qs=None, cu=C, lens=C + 4096, pos=None, KP=D, VP=E, table=C + 8192, O=None, os=None)

    def call(**kw):
        a = {**base, **kw}
        return lib.hf_paged_append(a["cache"], a["rope"], a["n"], a["K"], a["ks"], a["V"], a["vs"], a["Q"], a["qs"], a["cu"], a["lens"],
                                   a["pos"], a["KP"], a["VP"], a["table"], a["O"], a["os"], None)
    for name in ("cache", "K", "V", "cu", "lens", "KP", "VP", "table"):
        assert call(**{name: None}) == -1, name
    for name in ("K", "V", "KP", "VP"):
        assert call(**{name: base[name] + 8}) == -4, name
    for name in ("cu", "lens", "table", "pos"):
        assert call(**{name: C + 2}) == -4, name
    assert call(Q=F) == -1 and call(O=F) == -1
    assert call(ks=_strides(128, 60)) == -4
    assert call(VP=D + big - 256) == -2 and call(K=D + 256) == -2 and call(V=E) == -2 and call(Q=D, O=F) == -2 and call(Q=F, O=E) == -2
    assert call(Q=F, O=F + 128) == -2                                  # beside itself
    assert call(Q=F, O=F + 65536, os=_strides(64, 64)) == -2           # rows on top of each other
    assert call(n=0) == 0
    huge = ctypes.byref(_cache(n_pages=2147483647, heads=65535, heads_kv=65535, head_dim=128, dtype="f32", page_tokens=65536))
    assert call(cache=huge) == -2


def test_attention_arguments(lib):
    cache = _cache()
    need = hf.hf_paged_workspace_bytes(cache, 5)
    base = dict(cache=ctypes.byref(cache), Q=A, qs=None, n=5, cu=C, lens=C + 4096, KP=D, VP=E, table=C + 8192, O=F, os=None, lse=None,
                ws=1 << 30, size=need)

    def call(**kw):
        a = {**base, **kw}
        return lib.hf_paged_attn_fwd(a["cache"], a["Q"], a["qs"], a["n"], a["cu"], a["lens"], a["KP"], a["VP"], a["table"], a["O"], a["os"],
                                     a["lse"], a["ws"], a["size"], None)
    for name in ("cache", "Q", "cu", "lens", "KP", "VP", "table", "O"):
        assert call(**{name: None}) == -1, name
    for name in ("Q", "KP", "VP", "O"):
        assert call(**{name: base[name] + 8}) == -4, name
    for name in ("cu", "lens", "table", "lse"):
        assert call(**{name: C + 2}) == -4, name
    assert call(O=A) == -2 and call(O=A + 64) == -2 and call(O=D) == -2 and call(O=E + 128) == -2
    assert call(lse=F) == -2 and call(lse=D) == -2 and call(lse=A) == -2
    assert call(os=_strides(512, 32)) == -2 and call(qs=_strides(516, 64)) == -4
    if need:
        assert call(ws=None) == -5 and call(size=need - 1) == -5 and call(ws=(1 << 30) + 128) == -4
        assert call(ws=F) == -2 and call(ws=D) == -2
    assert call(n=0) == 0


def test_binding_takes_gpu_tensors_of_its_structures_only(lib):
    x = torch.zeros((4, 8, 64))
    pos = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(TypeError, match="GPU"):
        hf.hf_rope_axes_apply(hf.make_rope_axes([8]), x, pos, x)
    with pytest.raises(TypeError, match="hf_rope_axes"):
        hf.hf_rope_axes_apply(_cache(), x, pos, x)
    with pytest.raises(TypeError, match="hf_paged"):
        hf.hf_paged_attn_fwd(hf.make_rope_axes([8]), x, pos, pos, x, x, pos, x)
    with pytest.raises(hf.HFError):
        hf.hf_paged_append(_cache(heads_kv=3), x, x, pos, pos, x, x, pos)
