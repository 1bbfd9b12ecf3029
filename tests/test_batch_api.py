"""The batch calls refuse bad arguments before any HIP call (no GPU needed):
descriptors with made-up addresses, one fault each."""
import ctypes

import numpy as np
import pytest

from paper_2607_19547_amd import binding as b

BAD, UNS, SMALL = b.CS_ERR_INVALID_ARGUMENT, b.CS_ERR_UNSUPPORTED, b.CS_ERR_WORKSPACE_TOO_SMALL
PTR = 0x10000


def _geo(**kw):
    d = dict(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=128, sections=(16, 24, 24), dtype="bf16",
             chunk_start=[0, 64])
    d.update(kw)
    return b.Geo(**d)


def _pool(**kw):
    p = b._PagePool(PTR, 2 * PTR, 10)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _batch(**kw):
    c = b._Batch(3, 5, 4, 1, 0, *[PTR * i for i in range(1, 7)])
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _plan(**kw):
    c = b._PagePlan(*[PTR * i for i in range(1, 5)], 7, *[PTR * i for i in range(5, 10)])
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _rows(data=PTR, row=512, head=128):
    return b.Rows(data, row, head)


def _r(x):
    return None if x is None else ctypes.byref(x)


def _plan_call(geo=None, n_pages=10, batch=None, plan=None):
    return b.lib().batch_plan_pages((geo or _geo()).ref, n_pages, _r(batch or _batch()), _r(plan or _plan()), None)


def _append(geo=None, pool=None, layer=0, batch=None, q=None, k=None, v=None, out=None, eps=1e-6, wq=PTR, wk=PTR):
    return b.lib().qk_norm_rope_append((geo or _geo()).ref, _r(pool or _pool()), layer, _r(batch or _batch()),
                                       _r(q or _rows()), _r(k or _rows(2 * PTR)), _r(v or _rows(3 * PTR)), wq, wk, eps,
                                       _r(out or _rows(4 * PTR)), None)


def _attend(geo=None, pool=None, layer=0, batch=None, q=None, out=None, ws=PTR, ws_bytes=1 << 40):
    return b.lib().tree_attend_paged((geo or _geo()).ref, _r(pool or _pool()), layer, _r(batch or _batch()),
                                     _r(q or _rows()), _r(out or _rows(2 * PTR)), None, ws, ws_bytes, None)


def _commit(geo=None, pool=None, lb=0, le=2, batch=None, accepted=PTR, most=4, count=PTR, out=9 * PTR):
    return b.lib().tree_commit_paged((geo or _geo()).ref, _r(pool or _pool()), lb, le, _r(batch or _batch()), accepted,
                                     most, count, out, None)


def _says(word):
    assert word in b.lib().cs_last_error().decode(), b.lib().cs_last_error().decode()


@pytest.mark.parametrize("call", [_plan_call, _append, _attend, _commit])
@pytest.mark.parametrize("kw,code,word", [
    (dict(n_requests=-1), BAD, "negative"), (dict(n_rows=-1), BAD, "negative"), (dict(max_blocks=-2), BAD, "negative"),
    (dict(mask_words=-1), BAD, "negative"), (dict(max_rows=-1), BAD, "negative"),
    (dict(n_requests=4097), UNS, "4096"), (dict(row_start=None), BAD, "row_start"),
    (dict(cached_len=None), BAD, "cached_len"), (dict(block_table=None), BAD, "block_table"),
    (dict(mask_words=0), BAD, "mask_words"),
])
def test_bad_batch(built_lib, call, kw, code, word):
    assert call(batch=_batch(**kw)) == code
    _says(word)


@pytest.mark.parametrize("call", [_append, _attend, _commit])
@pytest.mark.parametrize("kw,word", [
    (dict(k_pages=None), "NULL"), (dict(v_pages=None), "NULL"), (dict(n_pages=0), "n_pages"),
    (dict(n_pages=1 << 25), "2^31"), (dict(n_pages=1 << 40), "2^31"), (dict(k_pages=PTR + 8), "16 bytes"),
    (dict(v_pages=PTR + 2), "16 bytes"),
])
def test_bad_pool(built_lib, call, kw, word):
    assert call(pool=_pool(**kw)) == BAD
    _says(word)


@pytest.mark.parametrize("call", [_plan_call, _append, _attend, _commit])
def test_bad_geometry_and_nulls(built_lib, call):
    assert call(geo=_geo(sections=(1, 2, 3))) == BAD
    _says("sum")
    L, g = b.lib(), _geo()
    assert L.batch_plan_pages(g.ref, 10, None, _r(_plan()), None) == BAD
    assert L.batch_plan_pages(g.ref, 10, _r(_batch()), None, None) == BAD
    assert L.qk_norm_rope_append(g.ref, None, 0, _r(_batch()), None, None, None, None, None, 0.0, None, None) == BAD
    assert L.tree_attend_paged(g.ref, _r(_pool()), 0, None, None, None, None, None, 0, None) == BAD


@pytest.mark.parametrize("call", [_append, _attend])
def test_bad_layer(built_lib, call):
    assert call(layer=2) == BAD and call(layer=-1) == BAD
    _says("layer")


@pytest.mark.parametrize("kw,word", [
    (dict(n_free=-1), "n_free"), (dict(free_pages=None), "NULL"), (dict(free_head=None), "NULL"),
    (dict(free_head_out=None), "NULL"), (dict(status=None), "NULL"), (dict(new_len=None), "NULL"),
    (dict(n_blocks=None), "NULL"), (dict(n_blocks_out=None), "NULL"),
    (dict(n_blocks_out=2 * PTR), "n_blocks_out"), (dict(free_head_out=5 * PTR), "free_head_out"),
])
def test_bad_plan(built_lib, kw, word):
    assert _plan_call(plan=_plan(**kw)) == BAD
    _says(word)


def test_plan_sizes_and_arrays(built_lib):
    assert _plan_call(n_pages=0) == BAD and _plan_call(n_pages=1 << 26) == BAD
    assert _plan_call(batch=_batch(slot=None)) == BAD and _plan_call(batch=_batch(coords=None)) == BAD
    assert _plan_call(batch=_batch(tree_mask=None, mask_words=0)) == BAD  # parents without a mask
    _says("tree mask")


@pytest.mark.parametrize("eps", [-1e-6, float("nan"), float("inf")])
def test_append_rejects_bad_eps(built_lib, eps):
    assert _append(eps=eps) == BAD
    _says("eps")


def test_append_rows(built_lib):
    for name in ("q", "k", "v", "out"):
        assert _append(**{name: b.Rows(None, 512, 128)}) == BAD
        _says("NULL")
        assert _append(**{name: _rows(row=-1)}) == BAD
        _says("stride")
    for row, head in ((512, 64), (100, 128), (256, 128), (0, 128), (512, 0)):  # written heads would overlap
        assert _append(out=_rows(4 * PTR, row, head)) == BAD
        _says("overlap")
    assert _append(q=_rows(PTR, 1024, 128), out=_rows(PTR, 512, 128)) == BAD  # in place, other strides
    _says("in place")
    assert _append(batch=_batch(slot=None)) == BAD and _append(batch=_batch(coords=None)) == BAD
    bad = b.Geo(2, 4, 2, 128, (16, 24, 24), "bf16", [0, 64], inv_freq=np.full(64, np.nan))
    assert _append(geo=bad) == BAD
    _says("finite")


def test_attend_rows_and_workspace(built_lib):
    assert _attend(q=b.Rows(None, 512, 128)) == BAD and _attend(out=b.Rows(None, 512, 128)) == BAD
    assert _attend(out=_rows(2 * PTR, 256, 128)) == BAD
    _says("overlap")
    assert _attend(q=_rows(PTR, 1024, 128), out=_rows(PTR, 512, 128)) == BAD
    n = ctypes.c_size_t(0)
    assert b.lib().tree_attend_paged_workspace(_geo().ref, _r(_batch()), None) == BAD
    assert b.lib().tree_attend_paged_workspace(_geo().ref, _r(_batch()), ctypes.byref(n)) == b.CS_OK
    if n.value:
        assert _attend(ws_bytes=n.value - 1) == SMALL and _attend(ws=None) == SMALL


@pytest.mark.parametrize("call", [_append, _attend])
def test_too_many_rows(built_lib, call):
    assert call(batch=_batch(n_rows=1 << 29)) == UNS
    _says("2^31")


def test_commit_arguments(built_lib):
    assert _commit(lb=1, le=0) == BAD and _commit(lb=-1) == BAD and _commit(le=3) == BAD
    assert _commit(most=-1) == BAD and _commit(accepted=None) == BAD and _commit(count=None) == BAD
    assert _commit(out=PTR) == BAD  # batch.cached_len
    _says("cached_len")


def test_nothing_to_do(built_lib):
    """Empty batches need no arrays and touch no device."""
    empty = b._Batch(0, 0, 0, 0, 0, None, PTR, None, None, None, None)
    none = b.Rows(None, 0, 0)
    assert _append(batch=empty, q=none, k=none, v=none, out=none) == b.CS_OK
    assert _attend(batch=empty, q=none, out=none, ws=None, ws_bytes=0) == b.CS_OK
    assert _commit(batch=empty, accepted=None, count=None, out=None) == b.CS_OK
    n = ctypes.c_size_t(1)
    assert b.lib().tree_attend_paged_workspace(_geo().ref, _r(empty), ctypes.byref(n)) == b.CS_OK and n.value == 0


def test_binding_checks_tensors(built_lib):
    """Types, shapes and memory are looked at before addresses are passed on."""
    torch = pytest.importorskip("torch")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    for args in ((i(2).long(), i(3), i(2, 4), i(5), i(5, 3)), (i(2), i(2), i(2, 4), i(5), i(5, 3)),
                 (i(2), i(3), i(3, 4), i(5), i(5, 3)), (i(2), i(3), i(2, 4), i(5), i(4, 3)),
                 (i(2), i(3), i(2, 8)[:, ::2], i(5), i(5, 3)), (i(2), i(3), i(2, 4), i(5), i(5, 3))):
        with pytest.raises(ValueError):  # the last one is right but for its memory: host tensors
            b.Batch(*args)
    with pytest.raises(ValueError):
        b.PagePool(_geo(), torch.zeros(3, 2, 2, 64, 128), torch.zeros(3, 2, 2, 64, 128))
    with pytest.raises(ValueError):
        b.Rows.of(torch.zeros(4, 2, 16)[..., ::2])
