"""The attention and the commit of a full batch: 4,096 requests, some without rows, some without a cache."""
import numpy as np
import pytest

from oracle import batch as ob
from tests.batch_util import Case, check_attend, tree, ancestors
from tests.test_gpu_tree_attention import _run

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

N = 4096


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.mark.parametrize("geo", [(2, 1, 128, "bf16"), (2, 1, 64, "bf16"), (1, 1, 16, "f32"), (1, 1, 80, "bf16")])
@pytest.mark.parametrize("trees", [False, True])
def test_attention(geo, trees):
    rng = np.random.default_rng(geo[2])
    cached, new = rng.integers(0, 30, N), rng.integers(0, 3, N)
    cached[[0, 1777, N - 1]], new[[0, 1777, N - 1]] = (700, 0, 2500), (40, 17, 9)
    new[100:200] = 0
    masks = sum([ancestors(tree(rng, int(n))) for n in new], []) if trees else None
    c = Case(1, cached.tolist(), new.tolist(), 16, *geo, masks=masks, layers=1, pad_rows=3)
    for max_rows in (1, 4000):
        out, lse = _run(c, 0, max_rows=max_rows)
        check_attend(c, 0, out, lse, f"{geo} max_rows {max_rows}")
        assert (out[c.rows:] == 7).all() and (lse[c.rows:] == 7).all()


def test_commit():
    from paper_2607_19547_amd import binding as b
    rng = np.random.default_rng(3)
    cached, new = rng.integers(0, 30, N), rng.integers(0, 6, N)
    c = Case(2, cached.tolist(), new.tolist(), 16, 1, 1, 16, "f32", layers=1)
    geo, pool, batch, _, _, _ = c.dev(b)
    acc = np.full((N, 5), -1)
    for i in range(N):
        rows = np.sort(rng.choice(5, rng.integers(0, 6), replace=False))  # (some are no rows of the request)
        acc[i, :len(rows)] = rows
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    count = rng.integers(0, 7, N)
    out = t(np.zeros(N))
    rk, rv = c.k.numpy().copy(), c.v.numpy().copy()
    want = ob.commit([rk, rv], (0, 1), cached, new, c.table.tolist(), acc, count)
    b.tree_commit_paged(geo, pool, 0, 1, batch, t(acc), t(count), out)
    assert out.tolist() == want
    assert np.array_equal(pool.tensors[0].cpu().numpy(), rk) and np.array_equal(pool.tensors[1].cpu().numpy(), rv)
