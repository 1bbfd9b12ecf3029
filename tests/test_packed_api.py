"""Refusals of the packed calls, before any HIP call (no GPU needed)."""
import ctypes

import numpy as np
import pytest

from paper_2607_19547_amd import binding as b

PTR = 0x10000
BAD, UNS, WS = b.CS_ERR_INVALID_ARGUMENT, b.CS_ERR_UNSUPPORTED, b.CS_ERR_WORKSPACE_TOO_SMALL


def _geo(d=128, p=64, layers=2, **kw):
    s = d // 2
    return b.Geo(layers, 4, 2, d, kw.pop("sections", (s - 2, 1, 1)), kw.pop("dtype", "bf16"), [0, p], **kw)


def _struct(cls, *a, **kw):
    s = cls(*a)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _pool(**kw):
    return _struct(b._PagePool, PTR, 2 * PTR, 10, **kw)


def _packed(**kw):
    return _struct(b._PackedPool, 3 * PTR, 10, **kw)


def _batch(**kw):
    return _struct(b._Batch, 3, 5, 4, 1, 0, *[PTR * i for i in range(1, 7)], **kw)


def _r(x):
    return None if x is None else ctypes.byref(x)


NONE = object()


def _pack(geo=None, pool=None, packed=None, lb=0, le=2, src=PTR, dst=PTR, n=3):
    pool, packed = (None if x is NONE else x or f() for x, f in ((pool, _pool), (packed, _packed)))
    return b.lib().pack_pages((geo or _geo()).ref, _r(pool), _r(packed), lb, le, src, dst, n, None)


def _unpack(geo=None, pool=None, packed=None, lb=0, le=2, src=PTR, dst=PTR, n=3, offsets=None):
    pool, packed = (None if x is NONE else x or f() for x, f in ((pool, _pool), (packed, _packed)))
    return b.lib().unpack_rebase_pages((geo or _geo()).ref, _r(packed), _r(pool), lb, le, src, dst, offsets, n, None)


def _attend(geo=None, pool=None, packed=None, layer=0, batch=None, blocks=PTR, sinks=0, window=0, q=None, out=None, ws=PTR,
            ws_bytes=1 << 40):
    pool, packed = (None if x is NONE else x or f() for x, f in ((pool, _pool), (packed, _packed)))
    rows = b.Rows(PTR, 512, 128)
    return b.lib().tree_attend_packed((geo or _geo()).ref, _r(pool), _r(packed), layer, _r(batch or _batch()), blocks,
                                      sinks, window, _r(q or rows), _r(out or b.Rows(2 * PTR, 512, 128)), None, ws,
                                      ws_bytes, None)


def _says(word):
    assert word in b.lib().cs_last_error().decode(), b.lib().cs_last_error().decode()


def test_page_bytes(built_lib):
    assert b.packed_page_bytes(_geo()) == 2 * 2 * 64 * 128 * 17 // 16
    assert b.packed_page_bytes(_geo(d=96, p=32, layers=7, dtype="f32")) == 7 * 2 * 32 * 96 * 17 // 16
    L, n = b.lib(), ctypes.c_size_t()
    assert L.packed_page_bytes(_geo().ref, None) == BAD
    assert L.packed_page_bytes(_geo(p=48).ref, ctypes.byref(n)) == UNS
    assert L.packed_page_bytes(_geo(d=80).ref, ctypes.byref(n)) == UNS
    assert L.packed_page_bytes(_geo(p=1 << 24).ref, ctypes.byref(n)) == UNS


@pytest.mark.parametrize("call", [_pack, _unpack, _attend])
@pytest.mark.parametrize("kw,word", [
    (dict(pool=NONE), "pool"), (dict(packed=NONE), "packed"), (dict(pool=_pool(k_pages=None)), "NULL"),
    (dict(pool=_pool(v_pages=2 * PTR + 4)), "16 bytes"), (dict(packed=_packed(pages=None)), "NULL"),
    (dict(packed=_packed(pages=PTR + 8)), "16 bytes"), (dict(packed=_packed(n_pages=0)), "n_pages"),
    (dict(packed=_packed(n_pages=1 << 25)), "2^31"), (dict(geo=_geo(sections=(1, 2, 3))), "sum"),
])
def test_bad_pools_and_geometry(built_lib, call, kw, word):
    assert call(**kw) == BAD
    _says(word)


@pytest.mark.parametrize("call", [_pack, _unpack, _attend])
@pytest.mark.parametrize("kw", [dict(p=48), dict(p=16), dict(d=80), dict(d=16, dtype="f32"), dict(p=1 << 24)])
def test_pages_that_cannot_be_packed(built_lib, call, kw):
    assert call(geo=_geo(**kw), pool=_pool(n_pages=1), packed=_packed(n_pages=1)) == UNS


@pytest.mark.parametrize("call", [_pack, _unpack])
@pytest.mark.parametrize("kw,word", [
    (dict(lb=-1), "layer_begin"), (dict(lb=2, le=1), "layer_begin"), (dict(le=3), "layer_begin"), (dict(n=-1), "n must"),
    (dict(src=None), "NULL"), (dict(dst=None), "NULL"),
])
def test_bad_entries(built_lib, call, kw, word):
    assert call(**kw) == BAD
    _says(word)


@pytest.mark.parametrize("call", [_pack, _unpack])
def test_nothing_to_do_and_too_much(built_lib, call):
    assert call(n=0, src=None, dst=None) == 0 and call(lb=1, le=1) == 0
    # 2^31 planes
    assert call(geo=_geo(layers=1 << 20), le=1 << 20, n=1 << 10) == UNS
    _says("2^31")


def test_unpack_frequencies(built_lib):
    assert _unpack(geo=b.Geo(2, 4, 2, 128, (62, 1, 1), "bf16", [0, 64], inv_freq=np.full(64, np.inf)), offsets=PTR) == BAD


@pytest.mark.parametrize("kw,code,word", [
    (dict(sinks=-1), BAD, "sinks"), (dict(window=-1), BAD, "window"), (dict(layer=2), BAD, "layer"),
    (dict(layer=-1), BAD, "layer"), (dict(ws=None), WS, "workspace"), (dict(ws_bytes=100), WS, "workspace"),
    (dict(q=b.Rows(None, 512, 128)), BAD, "q is NULL"), (dict(out=b.Rows(2 * PTR, 512, 64)), BAD, "overlap"),
    (dict(out=b.Rows(PTR, 1024, 128)), BAD, "in place"), (dict(out=b.Rows(2 * PTR, -1, 128)), BAD, "negative"),
    (dict(batch=_batch(n_requests=-1)), BAD, "negative"), (dict(batch=_batch(n_requests=4097)), UNS, "4096"),
    (dict(batch=_batch(cached_len=None)), BAD, "cached_len"), (dict(batch=_batch(mask_words=0)), BAD, "mask_words"),
    (dict(batch=_batch(max_blocks=1 << 27)), UNS, "2^31"), (dict(batch=_batch(n_rows=1 << 30)), UNS, "rows x heads"),
])
def test_bad_attention_arguments(built_lib, kw, code, word):
    assert _attend(**kw) == code
    _says(word)
    # with a window and no packed page too
    assert _attend(**dict(dict(window=5), **kw, packed=NONE, blocks=None)) == code
    _says(word)


def test_empty_batches_and_workspace(built_lib):
    assert _attend(batch=_batch(n_requests=0), ws=None) == 0 and _attend(batch=_batch(n_rows=0), ws=None) == 0
    L, n = b.lib(), ctypes.c_size_t()
    g = _geo()
    assert L.tree_attend_packed_workspace(g.ref, _r(_batch()), None) == BAD
    assert L.tree_attend_packed_workspace(g.ref, None, ctypes.byref(n)) == BAD
    assert L.tree_attend_packed_workspace(g.ref, _r(_batch(max_blocks=1 << 27)), ctypes.byref(n)) == UNS
    assert L.tree_attend_packed_workspace(g.ref, _r(_batch()), ctypes.byref(n)) == 0 and n.value > 0
    m = ctypes.c_size_t()
    assert L.tree_attend_paged_workspace(g.ref, _r(_batch()), ctypes.byref(m)) == 0 and n.value >= m.value
    for sizes in (dict(n_requests=9, n_rows=1000, max_blocks=77), dict(n_requests=1, n_rows=1, max_blocks=1)):
        assert L.tree_attend_packed_workspace(g.ref, _r(_batch(**sizes)), ctypes.byref(m)) == 0 and m.value == n.value
    assert L.tree_attend_packed_workspace(g.ref, _r(_batch(n_rows=0)), ctypes.byref(m)) == 0 and m.value == 0
