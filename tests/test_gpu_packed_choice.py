"""Which kernel a call of many rows with a window takes (bf16 x 128), off the library's trace: the window bounds what is
read, whatever the tables have room for, so the kernel for many rows is taken where it is the faster one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_19547_amd import binding
    return binding


def _taken(b, requests, cached, rows, sinks, window, packed, hq=16, hkv=2, page=64):
    """The kernels that a call launches; every page of the tables is one of a few."""
    geo = b.Geo(1, hq, hkv, 128, (16, 24, 24), "bf16", [0, page])
    blocks = -(-(cached + rows) // page)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    n = requests * rows
    kv = torch.zeros((4, 1, hkv, page, 128), dtype=torch.bfloat16, device="cuda")
    pool = b.PagePool(geo, kv, kv.clone())
    bits = b.PackedPool(geo, torch.zeros((4, b.packed_page_bytes(geo)), dtype=torch.uint8, device="cuda")) if packed else None
    batch = b.Batch(i32([cached] * requests), i32(np.arange(requests + 1) * rows),
                    i32(np.arange(requests * blocks).reshape(requests, blocks) % 4), i32(np.full(n, -1)),
                    i32(np.zeros((n, 3))), max_rows=rows)
    q = torch.zeros((n, hq, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(b.tree_attend_packed_workspace(geo, batch), dtype=torch.uint8, device="cuda")
    b.cs_trace_reset()
    b.cs_trace_only(None)
    b.cs_trace_enable(True)
    b.tree_attend_packed(geo, pool, bits, 0, batch, i32([cached // page] * requests) if packed else None, q,
                         torch.empty_like(q), None, ws, sinks=sinks, window=window)
    b.cs_trace_enable(False)
    got = set(b.cs_trace_collect())
    b.cs_trace_reset()
    return got


# requests, cached tokens, rows, window, packed: sizes at which the other kernel takes at least 1.25 times as long
MANY = [(1, 6001, 1950, 1024, False), (1, 6001, 1999, 1000, False), (1, 8192, 1950, 1024, True), (1, 8192, 1000, 1024, True),
        (1, 8192, 1000, 1024, False), (1, 8192, 1950, 256, True), (1, 8192, 500, 4096, False), (16, 8192, 64, 1024, False),
        (48, 8192, 16, 4096, False), (4, 8192, 250, 1024, True)]
FEW = [(1, 8192, 250, 256, False), (1, 8192, 64, 1024, True), (1, 8192, 64, 1024, False), (48, 8192, 4, 1024, True),
       (48, 8192, 4, 4096, True), (1, 8192, 16, 4096, False)]


@pytest.mark.parametrize("requests,cached,rows,window,packed", MANY)
def test_windows_of_many_rows(b, requests, cached, rows, window, packed):
    assert "packed_attend_wide" in _taken(b, requests, cached, rows, 4, window, packed)


@pytest.mark.parametrize("requests,cached,rows,window,packed", FEW)
def test_windows_of_few_rows(b, requests, cached, rows, window, packed):
    assert "packed_attend" in _taken(b, requests, cached, rows, 4, window, packed)


def test_filled_tables(b):
    assert "packed_attend_wide" in _taken(b, 1, 8192, 250, 0, 0, True)
