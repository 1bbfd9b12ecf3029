"""Scores and values that are not finite, seen by a row, wherever the cutting of the work puts them: alone in a
wavefront's tile, in a workgroup's piece, in a piece whose weight is too little for float32.

A score of NaN or +inf makes its row's outputs and log-sum-exp NaN; one of -inf is a key of weight 0, and a row whose
seen scores are all -inf gets NaN; an element that sees a value which is not finite is not finite.  Everything else
is held to the tolerances of batch_util."""
import copy

import numpy as np
import pytest

from tests.batch_util import Case, attend_tol, f64
from tests.test_gpu_tree_attention import _run

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FAST = [(16, 2, 128, "bf16"), (5, 5, 128, "bf16"), (12, 1, 64, "bf16"), (6, 2, 96, "bf16"), (2, 1, 256, "bf16"),
        (2, 2, 32, "bf16"), (8, 2, 128, "f32"), (3, 1, 64, "f32"), (4, 1, 32, "f32"), (4, 2, 16, "f32")]
ANY = [(2, 1, 80, "bf16"), (4, 4, 10, "f32")]
MAIN = [FAST[0], FAST[2], FAST[6], ANY[0]]


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _check(c, layer=1, ref_of=None, roomy=True):
    """Finite where the oracle is, within the tolerances; NaN rows (lse) equal; other elements not finite
    where the oracle's are not.  ref_of: the case that the oracle takes in the place of c."""
    out, lse = (f64(x) for x in _run(c, layer))
    ref, ref_lse, spread = (ref_of or c).attend_ref(layer)
    t_out, t_lse = attend_tol(ref, ref_lse, spread, c.dtype)
    what = f"{c.cached} + {c.new}, {c.hq}/{c.hkv} x {c.d} {c.dtype}"
    assert (np.isnan(lse) == np.isnan(ref_lse)).all(), f"{what}: NaN lost or made"
    assert np.isnan(out[np.isnan(ref_lse)]).all(), f"{what}: a row of NaN has outputs"
    fin = np.isfinite(ref)
    assert (np.isfinite(out) == fin).all(), f"{what}: {(np.isfinite(out) != fin).sum()} elements finite or not"
    assert np.isnan(out[np.isnan(ref)]).all(), f"{what}: NaN lost"
    inf = np.isinf(ref) & np.isinf(out)
    assert (out[inf] == ref[inf]).all(), f"{what}: an infinity's sign"
    assert (np.abs(out[fin] - ref[fin]) <= t_out[fin]).all(), f"{what}: off by {np.abs(out[fin] - ref[fin]).max():.3e}"
    ok = np.isfinite(ref_lse)
    assert (lse[~ok & ~np.isnan(ref_lse)] == ref_lse[~ok & ~np.isnan(ref_lse)]).all()
    assert (np.abs(lse[ok] - ref_lse[ok]) <= t_lse[ok]).all(), f"{what}: lse"
    if roomy and c.d == 128 and c.dtype == "bf16":  # with the kernel for many rows too
        _check(c.roomy(), layer, ref_of, roomy=False)


def _at(c, b, j):
    return c.table[b][j // c.page], slice(None), slice(None), j % c.page


@pytest.mark.parametrize("geo", FAST + ANY)
@pytest.mark.parametrize("new", [1, 5])
def test_own_key_alone_in_a_tile(geo, new):
    """One cached tile, and the row's own key in the next one."""
    cached = 16 if geo[3] == "f32" else 32
    c = Case(1, [cached, 64], [new, new], 16, *geo)
    c.k[_at(c, 0, cached)] = float("nan")  # row 0 of request 0, which all its rows see
    c.k[_at(c, 1, 64 + new - 1)] = float("nan")  # the last row of request 1, which it alone sees
    _check(c)


@pytest.mark.parametrize("geo", MAIN)
@pytest.mark.parametrize("new", [1, 6])
@pytest.mark.parametrize("first", [1024, 1111])
def test_pages_of_nan_fill_a_piece(geo, new, first):
    """768 keys in a row, more than the longest piece of a call with so few: whole tiles, and parts of them."""
    c = Case(2, [3000, 500], [new, new], 50 if geo in ANY else 16, *geo)
    for j in range(first, first + 768):
        c.k[_at(c, 0, j)] = float("nan")
    _check(c)


def _low_and_high(seed, new, geo, cached=3000, low=1500):
    """Scores of the first `low` keys 100 and more below the others', by natural logarithm: no float32 holds
    their weights.  Queries are positive and at least 1, keys -K and K throughout."""
    c = Case(seed, [cached], [new], 50 if geo in ANY else 16, *geo)
    c.q.copy_(c.q.abs() + 1.0)
    k = 64.0 / geo[2] ** 0.5  # the scores differ by 2 x k x sum(q) / sqrt(D) >= 128
    for j in range(cached + new):
        c.k[_at(c, 0, j)] = -k if j < low else k
    return c


@pytest.mark.parametrize("geo", MAIN)
@pytest.mark.parametrize("new", [1, 6])
def test_nan_score_far_below_the_others(geo, new):
    c = _low_and_high(3, new, geo)
    c.k[_at(c, 0, 700)] = float("nan")
    _check(c)


@pytest.mark.parametrize("geo", MAIN)
@pytest.mark.parametrize("new", [1, 6])
def test_values_that_are_not_finite_far_below_the_others(geo, new):
    c = _low_and_high(4, new, geo)
    c.v[_at(c, 0, 700)][..., 0] = float("inf")
    c.v[_at(c, 0, 701)][..., 1] = float("-inf")
    c.v[_at(c, 0, 702)][..., 2] = float("nan")
    _check(c)


@pytest.mark.parametrize("geo", FAST + ANY)
@pytest.mark.parametrize("new", [1, 6])
def test_scores_of_minus_infinity(geo, new):
    """Keys of weight 0, some of them filling pieces: as if they were not there."""
    c = Case(5, [3000, 40], [new, new], 50 if geo in ANY else 16, *geo)
    c.q.copy_(c.q.abs() + 0.1)
    page = c.page
    ref = copy.copy(c)
    ref.table = c.table.copy()
    for x in range(900 // page, 2000 // page):
        c.k[c.table[0][x]] = float("-inf")
        ref.table[0][x] = -1
    _check(c, ref_of=ref)


@pytest.mark.parametrize("geo", FAST + ANY)
def test_a_score_of_infinity(geo):
    """inf - inf: NaN for the rows that see it."""
    c = Case(7, [900, 40], [6, 6], 16, *geo)
    c.q.copy_(c.q.abs() + 0.1)
    c.k[_at(c, 0, 333)] = float("inf")
    c.k[_at(c, 1, 44)] = float("inf")
    _check(c)


@pytest.mark.parametrize("geo", FAST + ANY)
@pytest.mark.parametrize("new", [1, 6])
def test_only_scores_of_minus_infinity(geo, new):
    c = Case(6, [700, 40], [new, new], 16, *geo)
    c.q.copy_(c.q.abs() + 0.1)
    for x in range(-(-(700 + new) // 16)):
        c.k[c.table[0][x]] = float("-inf")
    _check(c)
