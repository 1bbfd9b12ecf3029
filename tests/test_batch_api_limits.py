"""Limits and contracts of the batch calls that the host decides (no GPU needed)."""
import ctypes
import os
import re

import pytest

from paper_2607_19547_amd import binding as b
from tests.test_batch_api import UNS, _attend, _batch, _geo, _r, _says


def _workspace(geo, batch):
    n = ctypes.c_size_t(0)
    return b.lib().tree_attend_paged_workspace(geo.ref, _r(batch), ctypes.byref(n)), n.value


@pytest.mark.parametrize("page,fits", [(64, 33_553_408), (1 << 20, 2047), (1, (1 << 31) - 65536)])
def test_attention_bounds_the_room_of_a_block_table(built_lib, page, fits):
    """Key indices, and those a few tiles ahead, stay below 2^31: the largest table that fits, and one block more."""
    geo = _geo(chunk_start=[0, page])
    assert fits * page <= (1 << 31) - 65536 < (fits + 1) * page
    assert _workspace(geo, _batch(max_blocks=fits))[0] == b.CS_OK
    for call in (lambda x: _workspace(geo, x)[0], lambda x: _attend(geo=geo, batch=x)):
        assert call(_batch(max_blocks=fits + 1)) == UNS
        _says("max_blocks")


@pytest.mark.parametrize("heads,d,dtype", [((16, 2), 128, "bf16"), ((4, 2), 64, "bf16"), ((4, 1), 256, "bf16"),
                                           ((8, 2), 128, "f32"), ((3, 1), 64, "f32"), ((4, 4), 16, "f32"), ((2, 1), 80, "bf16")])
def test_attention_workspace_is_the_geometrys(built_lib, heads, d, dtype):
    """One size for every batch: no change of its sizes or hints makes a workspace too small."""
    geo = _geo(n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=d, sections=(d // 2, 0, 0), dtype=dtype)
    sizes = {_workspace(geo, _batch(n_requests=n, n_rows=rows, max_blocks=blocks, max_rows=most, tree_mask=mask))
             for n in (1, 64, 4096) for rows in (1, 64, 5000) for blocks in (0, 8, 4096, 200_000) for most in (0, 1, 7, 4000)
             for mask in (None, 1 << 16)}
    assert len(sizes) == 1, sizes


def test_binding_refuses_a_mask_without_words(built_lib):
    """Its address is NULL, which the library takes for a batch without a mask."""
    torch = pytest.importorskip("torch")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="word"):
        b.Batch(i(2), i(3), i(2, 4), i(5), i(5, 3), torch.zeros(5, 0, dtype=torch.int64))


def test_exports_are_the_headers(built_lib):
    """The binding names every function that the header declares, and the library has each."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "chronostitch.h")
    with open(path) as f:
        names = re.findall(r"^(?:cs_status|const char\*|int32_t|void) (\w+)\(", f.read(), re.M)
    assert len(names) > 20 and sorted(b.EXPORTS) == sorted(names)
    assert all(hasattr(b.lib(), name) for name in names)
