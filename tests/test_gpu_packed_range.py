"""Float32 queries at the ends of their range over packed pages: the three bf16 terms of a query hold every finite
magnitude from 2^-110 on with all its bits."""
import numpy as np
import pytest

from tests.batch_util import f64
from tests.packed_util import PackedCase, check, row_hints, tol

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# instances of row tiles of 16 to 32 with one and two tiles a step, and one without an instance
GEOS = [(8, 2, 128, "f32"), (3, 1, 64, "f32"), (4, 1, 32, "f32"), (4, 2, 224, "f32")]
MOST = float(np.finfo(np.float32).max)
BORDER = float(np.uint32(0x7F7F8000).view(np.float32))  # from here on a magnitude rounds to infinity in bf16


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.fixture(scope="module")
def b(built_lib):
    from paper_2607_19547_amd import binding
    return binding


def _case(seed, geo, least, **kw):
    """Keys whose blocks' powers of two are 2^least to 2^(least + 3), in ordinary pages of that size too."""
    d = geo[2]
    c = PackedCase(seed, [12, 1], [12 * 32 + 3, 40], [3, 1], 32, *geo, **kw)
    n, s = 16 * d, d
    x = c.bits.reshape(c.n4, c.layers * geo[1], -1)
    x[:, :, n:n + s] = c.rng.integers(127 + least, 127 + least + 4, (c.n4, c.layers * geo[1], s))
    c.k = c.k.sign() * (c.k.abs() + 0.5) * 2.0 ** (least + 2)  # (none below the least normal number)
    return c


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("masked", [False, True])
def test_queries_near_the_largest_number(b, geo, masked):
    """An element of every query is as large as float32 has them; the keys are so small that scores are ordinary."""
    kw = dict(masks=[1, 3, 5, 1]) if masked else {}
    c = _case(31, geo, -125, **kw)
    hq, d = geo[0], geo[2]
    large = [MOST, -MOST, BORDER, -BORDER, float(np.nextafter(np.float32(BORDER), np.float32(0)))]
    for r in range(c.rows):
        for h in range(hq):
            c.q[r, h, int(c.rng.integers(d))] = large[(r * hq + h) % len(large)]
    check(c, b)


@pytest.mark.parametrize("geo", GEOS)
def test_small_queries(b, geo):
    """Queries of 2^-118 and keys of 2^114: the terms go down to 2^-133, below the least normal bf16 number (2^-126), so
    what they lose of an element is at most 2^-134, 2^-16 of it.  (Terms flushed at 2^-126 would lose 2^-8.)  All are
    positive, so that losses add up and show in lse."""
    c = _case(32, geo, 114)
    c.bits.reshape(c.n4, c.layers * geo[1], -1)[:, :, :16 * geo[2]] &= 0x77
    c.k = c.k.abs()
    c.q = torch.from_numpy((c.rng.uniform(1, 2, tuple(c.q.shape)) * 2.0 ** -118).astype(np.float32))
    ref, ref_lse, spread = c.attend_ref(1)
    t, t_lse = tol(ref, ref_lse, spread, "f32")
    lost = 2.0 ** -16 * spread[..., geo[2]]  # of a score, whose magnitudes' sum is at most that entry
    t, t_lse = t + spread[..., :geo[2]] * 2 * lost[..., None], t_lse + lost
    for hint in row_hints(c):
        out, lse = c.run(b, max_rows=hint)
        assert (np.abs(f64(out) - ref) <= t).all(), f"max_rows {hint}: off by {np.abs(f64(out) - ref).max():.3e}"
        assert (np.abs(f64(lse) - ref_lse) <= t_lse).all(), f"max_rows {hint}: lse"
