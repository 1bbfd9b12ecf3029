"""Whole numbers that 32 bits do not hold are refused by the binding, before anything else (no GPU needed): passed on,
their low bits would count as another number."""
import types

import pytest

from paper_2607_19547_amd import binding as b

LARGE = [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 64 + 1, -2 ** 31 - 1, -2 ** 32]


@pytest.fixture(scope="module")
def geo(built_lib):
    return b.Geo(2, 16, 2, 128, (16, 24, 24), "bf16", [0, 64])


def _tensor(*shape):
    return types.SimpleNamespace(shape=shape)


@pytest.mark.parametrize("x", LARGE)
@pytest.mark.parametrize("name", ["layer", "sinks", "window"])
def test_packed_attention(geo, name, x):
    kw = dict(dict(layer=0, sinks=0, window=0), **{name: x})
    with pytest.raises(ValueError, match=name):
        b.tree_attend_packed(geo, None, None, kw["layer"], None, None, None, None, sinks=kw["sinks"], window=kw["window"])


@pytest.mark.parametrize("x", LARGE)
def test_layers_of_pages(geo, x):
    page = types.SimpleNamespace(c=b._PagePool(), device=0, geo=geo)
    packed = types.SimpleNamespace(c=b._PackedPool(), device=0, geo=geo)
    for begin, end, name in ((x, 1, "layer_begin"), (0, x, "layer_end")):
        with pytest.raises(ValueError, match=name):
            b.pack_pages(geo, page, packed, begin, end, _tensor(1), None)
        with pytest.raises(ValueError, match=name):
            b.unpack_rebase_pages(geo, packed, page, begin, end, _tensor(1), None)
        with pytest.raises(ValueError, match=name):
            b.tree_commit_paged(geo, page, begin, end, types.SimpleNamespace(c=b._Batch(), device=0), None, None)
    if x > 0:
        with pytest.raises(ValueError, match="n must"):
            b.pack_pages(geo, page, packed, 0, 1, _tensor(x), None)
        with pytest.raises(ValueError, match="n must"):
            b.unpack_rebase_pages(geo, packed, page, 0, 1, _tensor(x), None)


@pytest.mark.parametrize("x", LARGE)
def test_layers_elsewhere(geo, x):
    batch, pool = types.SimpleNamespace(c=b._Batch(), device=0), types.SimpleNamespace(c=b._PagePool(), device=0, geo=geo)
    with pytest.raises(ValueError, match="layer "):
        b.tree_attend_paged(geo, pool, x, batch, None, None)
    with pytest.raises(ValueError, match="layer "):
        b.qk_norm_rope_append(geo, pool, x, batch, None, None, None, None)
    with pytest.raises(ValueError, match="n_layers_per_call"):
        b.selective_attend_scatter_workspace(geo, 1, x)
    with pytest.raises(ValueError, match="score_layer"):
        b.score_deviation_topk(geo, None, x, None, 0.5, None, None)
    with pytest.raises(ValueError, match="layer_begin"):
        b.selective_attend_scatter(geo, None, None, x, 1, None, 1, None, None, None, None)


@pytest.mark.parametrize("x", LARGE)
def test_hint_of_a_batch(x):
    with pytest.raises(ValueError, match="max_rows"):
        b.Batch(_tensor(1), _tensor(2), _tensor(1, 1), _tensor(1), _tensor(1, 3), max_rows=x)


def test_ends_of_the_range(geo):
    assert b._int32(2 ** 31 - 1, "x") == 2 ** 31 - 1 and b._int32(-2 ** 31, "x") == -2 ** 31
