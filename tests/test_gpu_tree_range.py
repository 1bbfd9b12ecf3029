"""Values near the ends of float32's range, in requests that are cut into pieces and in whole ones: the same
results, within the tolerances of batch_util (without their absolute part)."""
import numpy as np
import pytest

from tests.batch_util import Case, attend_tol, f64
from tests.test_gpu_tree_attention import _run
from tests.test_gpu_tree_nonfinite import _low_and_high

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

GEOS = [(16, 2, 128, "bf16"), (12, 1, 64, "bf16"), (8, 2, 128, "f32"), (2, 1, 80, "bf16")]


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _check(c, roomy=True):
    out, lse = (f64(x) for x in _run(c))
    ref, ref_lse, spread = c.attend_ref(1)
    t_out, t_lse = attend_tol(ref, ref_lse, spread, c.dtype)
    d = np.abs(out - ref)
    assert (d <= t_out - 1e-30).all(), f"{c.hq}/{c.hkv} x {c.d} {c.dtype}: off by up to {(d / np.abs(ref)).max():.3e} of it"
    assert (np.abs(lse - ref_lse) <= t_lse).all()
    if roomy and c.d == 128 and c.dtype == "bf16":  # with the kernel for many rows too
        _check(c.roomy(), roomy=False)


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("cached,new", [(5000, 40), (5000, 3), (60, 40)])
def test_large_values(geo, cached, new):
    """One key with nearly all of the weight and values of 2^122 to 2^123, beside values of about 1."""
    c = Case(1, [cached], [new], 16, *geo)
    c.q.copy_(c.q.abs() + 1.0)
    c.k.mul_(0.01)
    j = cached * 4 // 9
    page, off = c.table[0][j // 16], j % 16
    c.k[page, :, :, off] = 64.0 / geo[2] ** 0.5  # a score of at least 64, of the others at most a few
    v = c.v[page, :, :, off]
    v.copy_(torch.sign(v) * (1 + torch.rand(v.shape, generator=torch.Generator().manual_seed(0))) * 2.0 ** 122)
    _check(c)


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("cached,new", [(5000, 40), (5000, 3), (60, 40)])
def test_small_values(geo, cached, new):
    """Values of 2^-120 to 2^-119, weights alike (so that the products stay normal floats)."""
    c = Case(2, [cached], [new], 16, *geo, std_q=0.1)
    c.v.copy_((1 + torch.rand(c.v.shape, generator=torch.Generator().manual_seed(0))) * 2.0 ** -120)
    _check(c)


@pytest.mark.parametrize("geo", GEOS[:3])
@pytest.mark.parametrize("new", [1, 6])
def test_large_values_far_below_the_others(geo, new):
    """Values of 2^110 behind scores so far below that they count for nothing (3,000 x 2^110 x e^-128 at most)."""
    c = _low_and_high(3, new, geo, low=2999)
    for j in range(2999):
        page, off = c.table[0][j // 16], j % 16
        c.v[page, :, :, off] = 2.0 ** 110
    _check(c)
