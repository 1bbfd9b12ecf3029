"""qk_norm_rope_append on the GPU against the float64 oracle.

Tolerance, element by element.  With c, s off by 2^-24 each (float64 angles
rounded once), the norm's factor by (D + 8) 2^-24 relative (a float32 sum of D
squares, a square root, a division) and four more float32 roundings, an
element is off by at most (D + 16) 2^-24 of its pair's norm; the output is
rounded once: 2^-8 of it in bf16, 2^-24 in float32."""
import numpy as np
import pytest

from oracle import batch as ob
from tests.batch_util import f64, rnd, sections, theta
from tests.gpu_util import pair_norm

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _t(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def _check(got, ref, dtype):
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = (ref.shape[-1] + 16) * 2.0 ** -24 * pair_norm(ref) * (1 + half) + half * np.abs(ref) + 1e-37
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, by up to {np.abs(got - ref).max():.3e}"


class Case:
    def __init__(self, seed, rows, hq, hkv, d, dtype, page=16, layers=2, pad=0, layout="fused", weights=True, far=100_000):
        from paper_2607_19547_amd import binding as b
        g = self.g = np.random.default_rng(seed)
        self.b, self.dtype, self.rows, self.hq, self.hkv, self.d, self.page = b, dtype, rows, hq, hkv, d, page
        n = self.n = rows + pad
        if layout == "fused":
            x = rnd(g, (n, hq + 2 * hkv, d), dtype, 1.7).cuda()
            self.q, self.k, self.v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        elif layout == "heads":  # [H][n][D]
            self.q, self.k, self.v = (rnd(g, (h, n, d), dtype, 1.7).cuda().transpose(0, 1) for h in (hq, hkv, hkv))
        else:  # odd: an element before every row, so that nothing is aligned
            self.q, self.k, self.v = (rnd(g, (n, h * d + 1), dtype, 1.7).cuda()[:, 1:].unflatten(1, (h, d))
                                      for h in (hq, hkv, hkv))
        self.w = [rnd(g, (d,), dtype).cuda().add_(1.0) if weights else None for _ in range(2)]
        n_pages = -(-n // page) + 3
        self.slots = g.permutation(n_pages * page)[:n]
        self.coords = np.stack([g.integers(-50, far, n), g.integers(-32, 32, n), g.integers(0, 32, n)], 1)
        self.kp, self.vp = (rnd(g, (n_pages, layers, hkv, page, d), dtype).cuda() for _ in range(2))
        self.geo = b.Geo(layers, hq, hkv, d, sections(d), dtype, [0, page])
        self.pool = b.PagePool(self.geo, self.kp, self.vp)
        self.batch = b.Batch(_t([0]), _t([0, rows]), _t([[0]]), _t(self.slots), _t(self.coords))
        self.q_out = torch.full((n, hq, d), 7.0, dtype=self.q.dtype, device="cuda")

    def ref(self, layer, eps):
        sec, th, co = sections(self.d), theta(self.d), self.coords[:self.rows]
        w = [None if x is None else f64(x) for x in self.w]
        q = ob.norm_rope(f64(self.q[:self.rows]), w[0], eps, co, sec, th)
        k = ob.norm_rope(f64(self.k[:self.rows]), w[1], eps, co, sec, th)
        return q, k, f64(self.v[:self.rows])

    def run(self, layer=1, eps=1e-6, q_out=None, **kw):
        self.b.qk_norm_rope_append(self.geo, self.pool, layer, self.batch, self.q, self.k, self.v,
                                   self.q_out if q_out is None else q_out, *self.w, eps, **kw)

    def check(self, layer=1, eps=1e-6):
        kp, vp = f64(self.kp), f64(self.vp)
        q, k, v = self.ref(layer, eps)
        self.run(layer, eps)
        torch.cuda.synchronize()
        _check(f64(self.q_out[:self.rows]), q, self.dtype)
        assert (self.q_out[self.rows:] == 7.0).all()
        pg, off = self.slots[:self.rows] // self.page, self.slots[:self.rows] % self.page
        got_k, got_v = f64(self.kp), f64(self.vp)
        _check(got_k[pg, layer, :, off], k, self.dtype)
        assert np.array_equal(got_v[pg, layer, :, off], v)
        for got, was in ((got_k, kp), (got_v, vp)):  # everything else is as it was
            got[pg, layer, :, off] = was[pg, layer, :, off]
            assert np.array_equal(got, was)


@pytest.mark.parametrize("rows", [1, 5, 67])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 2, 128, "bf16"), (7, 7, 64, "bf16"), (12, 1, 128, "f32"), (4, 2, 16, "f32"),
                                            (6, 3, 96, "bf16"), (2, 1, 80, "f32"), (3, 1, 2, "f32"), (2, 2, 10, "bf16"),
                                            (2, 1, 512, "bf16"), (2, 1, 512, "f32"), (5, 5, 256, "bf16"), (4, 1, 16, "bf16"),
                                            (2, 1, 8, "f32")])
def test_against_the_oracle(rows, hq, hkv, d, dtype):
    Case(rows, rows, hq, hkv, d, dtype, pad=rows // 2).check()


@pytest.mark.parametrize("layout", ["heads", "odd"])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (128, "f32"), (64, "bf16"), (40, "bf16")])
def test_layouts(layout, d, dtype):
    Case(1, 37, 8, 2, d, dtype, page=7, layout=layout).check(layer=0)


def test_without_norm_and_large_rows():
    Case(2, 33, 16, 2, 128, "bf16", weights=False).check()
    Case(3, 6000, 16, 2, 128, "bf16", page=64).check()
    Case(4, 700, 4, 4, 128, "f32", page=48, far=(1 << 31) - 1).check()  # coordinates up to the largest


def test_room_for_many_rows():
    """Row arrays with much room: another way of loading, the rows of the step alone."""
    Case(9, 5, 16, 2, 128, "bf16", page=64, pad=13_500).check()
    Case(10, 3, 4, 4, 128, "f32", page=64, pad=11_000).check()


def test_in_place_queries_and_one_side_normed():
    c = Case(5, 21, 16, 2, 128, "bf16")
    c.w[1] = None
    q, k, _ = c.ref(1, 0.0)
    c.run(eps=0.0, q_out=c.q)
    _check(f64(c.q), q, "bf16")
    pg, off = c.slots // c.page, c.slots % c.page
    _check(f64(c.kp)[pg, 1, :, off], k, "bf16")


def test_rows_without_a_slot():
    c = Case(6, 9, 4, 2, 128, "bf16")
    before = f64(c.kp)
    slots = c.slots.copy()
    slots[[1, 4, 7]] = [-1, 1 << 30, c.kp.shape[0] * c.page]
    c.batch.tensors[3].copy_(_t(slots))
    q, _, v = c.ref(1, 1e-6)
    c.run()
    _check(f64(c.q_out), q, "bf16")
    keep = [0, 2, 3, 5, 6, 8]
    pg, off = slots[keep] // c.page, slots[keep] % c.page
    assert np.array_equal(f64(c.vp)[pg, 1, :, off], v[keep])
    after = f64(c.kp)
    after[pg, 1, :, off] = before[pg, 1, :, off]
    assert np.array_equal(after, before)


def test_zero_rows_and_zero_heads_of_values():
    c = Case(7, 4, 4, 2, 128, "bf16")
    c.q.zero_()  # a zero head stays zero: 0 / sqrt(eps)
    c.run()
    assert (c.q_out == 0).all()
    c.batch.tensors[1].copy_(_t([0, 0]))  # the step has no rows
    before = c.kp.clone()
    c.q_out.fill_(3.0)
    c.k.fill_(1.0)
    c.run()
    assert torch.equal(before, c.kp) and (c.q_out == 3.0).all()


def test_another_stream_and_a_captured_graph():
    c = Case(8, 19, 16, 2, 128, "bf16")
    c.run()
    torch.cuda.synchronize()
    q, k = c.q_out.clone(), c.kp.clone()
    c.q_out.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(c.q_out, q) and torch.equal(c.kp, k)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for _ in range(3):
        c.q_out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.q_out, q) and torch.equal(c.kp, k)
