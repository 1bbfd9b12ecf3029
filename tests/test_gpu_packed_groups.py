"""Query heads per KV head that do not divide a row tile (7, 5, 12, 3): a row's heads lie in two row tiles, whose spans,
clear tiles, lengths and merges then begin and end inside a row."""
import numpy as np
import pytest

from tests.batch_util import ancestors, tree
from tests.packed_util import PackedCase, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# bf16 x 128 has the kernel for many rows (row tiles of 256), the others row tiles of 32 and 64
WIDE = [(28, 4, 128, "bf16"), (5, 1, 128, "bf16"), (12, 1, 128, "bf16")]
GEOS = WIDE + [(7, 1, 64, "bf16"), (5, 1, 96, "bf16"), (3, 1, 64, "f32")]


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.fixture(scope="module")
def b(built_lib):
    from paper_2607_19547_amd import binding
    return binding


def _rows(geo, tiles):
    """Rows that take so many row tiles of 256, and a part of one more."""
    return 256 * tiles * geo[1] // geo[0] + 5


def test_rows_lie_in_two_row_tiles():
    """(what the sizes below are for)"""
    for geo in GEOS:
        assert 256 % (geo[0] // geo[1]) and 32 % (geo[0] // geo[1])


@pytest.mark.parametrize("geo", GEOS)
def test_many_rows(b, geo):
    check(PackedCase(41, [9, 1], [9 * 32 + 11, 40], [_rows(geo, 2), 9], 32, *geo, layers=1), b, 0)


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("sinks,window", [(0, 1), (4, 40), (37, 64), (70, 130), (500, 500)])
def test_windows(b, geo, sinks, window):
    """Windows that begin inside a tile for one row of a row tile and behind it for the next."""
    check(PackedCase(42, [20, 2], [700, 90], [_rows(geo, 2), 33], 32, *geo, sinks=sinks, window=window, layers=1), b, 0)


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("sinks,window", [(0, 2), (33, 50), (45, 9)])
def test_windows_of_trees(b, geo, sinks, window):
    rng = np.random.default_rng(43)
    new = [_rows(geo, 1), 30]
    masks = [m for n in new for m in ancestors(tree(rng, n, 2))]
    check(PackedCase(43, [9, 0], [32 * 9 + 3, 3], new, 32, *geo, sinks=sinks, window=window, masks=masks, layers=1), b, 0)


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("page", [16, 48])
def test_behind_ordinary_pages(b, geo, page):
    check(PackedCase(44, None, [500, 0], [_rows(geo, 1), 60], page, *geo, sinks=4, window=100, layers=1), b, 0)


@pytest.mark.parametrize("geo", WIDE)
def test_merged_pieces(b, geo):
    """Long enough that row tiles are cut into pieces."""
    for window in (0, 1500):
        check(PackedCase(45, [150], [150 * 32 + 9], [_rows(geo, 1)], 32, *geo, sinks=70, window=window, layers=1), b, 0)


@pytest.mark.parametrize("geo", [WIDE[0], GEOS[4]])
def test_nan_blocks(b, geo):
    """A NaN block of values reaches the rows that see it, whichever row tile their heads lie in."""
    hq, hkv, d, _ = geo
    c = PackedCase(46, [8], [8 * 32 + 7], [_rows(geo, 1)], 32, *geo, sinks=5, window=70, layers=1)
    n, s = 16 * d, d
    for blk in (0, 6, 7):
        c.bits.reshape(c.n4, hkv, -1)[c.table[0, blk], 0, 2 * n + s + 9 + blk] = 255
    check(c, b, 0)
