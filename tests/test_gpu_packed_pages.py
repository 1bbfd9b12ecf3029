"""Pages into 4 bits and back.  Packing is exact: bytes are compared with the oracle's.  Restored keys are the codes'
values, turned; values and keys that stay where they are come back bit by bit."""
import numpy as np
import pytest

from oracle import packed as op
from tests.batch_util import f64, sections, theta

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# layers, KV heads, page, head dim, type: planes smaller than a workgroup's share, larger, and no multiple of it
SHAPES = [(2, 2, 64, 128, "bf16"), (3, 1, 32, 32, "bf16"), (1, 5, 96, 64, "bf16"), (2, 1, 160, 96, "bf16"),
          (1, 2, 256, 256, "bf16"), (1, 1, 32, 512, "bf16"), (1, 3, 32, 160, "bf16"), (2, 2, 64, 64, "f32"),
          (1, 3, 32, 128, "f32"), (1, 1, 96, 224, "f32"), (7, 3, 32, 32, "f32"), (1, 1, 512, 128, "bf16")]


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.fixture(scope="module")
def b(built_lib):
    from paper_2607_19547_amd import binding
    return binding


def _geo(b, layers, hkv, p, d, dtype):
    return b.Geo(layers, 2 * hkv, hkv, d, sections(d), dtype, [0, p])


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _t(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _wild(rng, shape, dtype):
    """Magnitudes from 2^-40 to 2^40 by row, ties, zeros, numbers below the least normal one, a few not finite."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-40, 41, shape[:-1] + (1,))
    x = np.where(rng.random(shape) < 0.1, np.sign(x) * 2.0 ** rng.integers(-3, 3, shape) * rng.choice([1.0, 1.25, 1.5, 1.75],
                                                                                                      shape), x)
    x = np.where(rng.random(shape) < 0.05, 0.0 * x, x)
    x[0, ..., 3, :] *= 1e-38 / np.abs(x[0, ..., 3, :]).max()
    x[0, ..., 4, :] = np.sign(x[0, ..., 4, :]) * 2.0 ** rng.integers(-140, -110, x[0, ..., 4, :].shape)
    x[0, ..., 5, :] *= 3.3e38 / np.abs(x[0, ..., 5, :]).max()
    x[0, ..., 6, :] = 0
    x[0, 0, 0, 7, 1], x[0, 0, 0, 8, 2], x[0, 0, 0, 9, 3] = np.inf, np.nan, -np.inf
    return torch.from_numpy(x.astype(np.float32)).to(_dt(dtype))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("wild", [False, True])
def test_pack_is_exact(b, shape, wild):
    layers, hkv, p, d, dtype = shape
    rng = np.random.default_rng(p + d + wild)
    full = (3, layers, hkv, p, d)
    k, v = ((_wild(rng, full, dtype) if wild else torch.from_numpy(rng.standard_normal(full, dtype=np.float32)).to(_dt(dtype)))
            for _ in range(2))
    geo = _geo(b, *shape)
    assert b.packed_page_bytes(geo) == layers * hkv * op.plane_bytes(p, d)
    pages = torch.full((4, b.packed_page_bytes(geo)), 0xa5, dtype=torch.uint8, device="cuda")
    b.pack_pages(geo, b.PagePool(geo, k.cuda(), v.cuda()), b.PackedPool(geo, pages), 0, layers, _t([2, 0]), _t([3, 1]))
    got = pages.cpu().numpy()
    want = op.encode(f64(k)[[0, 2]], f64(v)[[0, 2]])
    assert (got[[0, 2]] == 0xa5).all(), "pages that are no destination"
    assert (got[[1, 3]] == want).all(), f"{(got[[1, 3]] != want).sum()} bytes of {want.size} differ"


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[4], SHAPES[7]])
def test_layers_entries_and_neighbours(b, shape):
    """A range of layers, entries outside the pools, one source twice; everything else stays as it is."""
    layers, hkv, p, d, dtype = (3,) + shape[1:]
    rng = np.random.default_rng(1)
    geo = _geo(b, layers, hkv, p, d, dtype)
    k, v = (torch.from_numpy(rng.standard_normal((4, layers, hkv, p, d), dtype=np.float32)).to(_dt(dtype)) for _ in range(2))
    n = b.packed_page_bytes(geo)
    pages = torch.full((5, n), 0x11, dtype=torch.uint8, device="cuda")
    pool, packed = b.PagePool(geo, k.cuda(), v.cuda()), b.PackedPool(geo, pages)
    b.pack_pages(geo, pool, packed, 1, 2, _t([1, -1, 4, 2, 2, 1]), _t([4, 0, 1, 5, 2, 0]))
    want = np.full((5, layers, n // layers), 0x11, np.uint8)
    for s, z in ((1, 4), (2, 2), (1, 0)):
        want[z, 1] = op.encode(f64(k)[s:s + 1, 1:2], f64(v)[s:s + 1, 1:2]).reshape(-1)
    assert (pages.cpu().numpy().reshape(want.shape) == want).all()
    # and back, into a pool that holds a pattern
    ko, vo = torch.full_like(pool.tensors[0], 9.0), torch.full_like(pool.tensors[1], -9.0)
    b.unpack_rebase_pages(geo, packed, b.PagePool(geo, ko, vo), 1, 2, _t([4, 7, 2, -2]), _t([3, 0, 0, 1]))
    dk, dv = op.decode(want.reshape(5, -1)[[4, 2]], layers, hkv, p, d)
    rk, rv = np.full(k.shape, 9.0), np.full(k.shape, -9.0)
    rk[[3, 0], 1], rv[[3, 0], 1] = dk[:, 1], dv[:, 1]
    assert (f64(ko) == rk).all() and (f64(vo) == rv).all()
    # nothing to do
    b.pack_pages(geo, pool, packed, 1, 1, _t([0]), _t([0]))
    b.pack_pages(geo, pool, packed, 0, 3, _t([]), _t([]))
    b.unpack_rebase_pages(geo, packed, pool, 0, 3, _t([]), _t([]), torch.zeros((0, 3), dtype=torch.int32, device="cuda"))
    assert (pages.cpu().numpy().reshape(want.shape) == want).all()


def _turned(k, off, d, p_sections):
    axis = np.repeat(np.arange(3), p_sections)
    a = np.asarray(off, np.float64)[axis] * theta(d)
    c, s, x, y = np.cos(a), np.sin(a), k[..., :d // 2], k[..., d // 2:]
    return np.concatenate([x * c - y * s, x * s + y * c], -1), np.concatenate([np.hypot(x, y)] * 2, -1)


@pytest.mark.parametrize("shape", SHAPES)
def test_restore_and_turn(b, shape):
    layers, hkv, p, d, dtype = shape
    rng = np.random.default_rng(p * d)
    geo = _geo(b, *shape)
    n = 20 if p * d <= 2048 else 4  # (several entries in a workgroup where planes are small)
    s, c = p * d // 32, p * d // 2
    bits = rng.integers(0, 256, (n, layers * hkv, 2 * (s + c)), dtype=np.uint8)
    for a in (c, 2 * c + s):
        bits[:, :, a:a + s] = rng.integers(110, 140, (n, layers * hkv, s))
    bits = bits.reshape(n, -1)
    off = rng.integers(-200_000, 200_000, (n, 3)).astype(np.int32)
    off[1] = 0
    off[2] = (0, 0, 7)
    off[3] = (2 ** 31 - 1, -2 ** 31, 5)
    src, dst = rng.permutation(n), rng.permutation(n)
    ko, vo = (torch.zeros((n, layers, hkv, p, d), dtype=_dt(dtype), device="cuda") for _ in range(2))
    b.unpack_rebase_pages(geo, b.PackedPool(geo, torch.from_numpy(bits).cuda()), b.PagePool(geo, ko, vo), 0, layers, _t(src),
                          _t(dst), torch.from_numpy(off).cuda())
    dk, dv = op.decode(bits, layers, hkv, p, d)
    gk, gv = f64(ko), f64(vo)
    assert (gv[dst] == dv[src]).all()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for i in range(n):
        if not off[i].any():
            assert (gk[dst[i]] == dk[src[i]]).all()
            continue
        want, pair = _turned(dk[src[i]], off[i], d, sections(d))
        # cos and sin rounded to float32 (2^-24 each of the pair's length), two products and a sum in float32 (three
        # roundings), the angle's own error in float64 (2^-53 of 2^31 x theta, reduced: 2^-21 at most), one to the type
        t = pair * (5 * 2.0 ** -24 + 2.0 ** -21) * (1 + half) + half * np.abs(want) + 1e-30
        assert (np.abs(gk[dst[i]] - want) <= t).all(), f"{shape} entry {i}: off by {np.abs(gk[dst[i]] - want).max():.3e}"


def test_nan_blocks_and_limits(b):
    """A block that is NaN comes back as NaN and no other one; the turn takes it to its pairs' elements."""
    layers, hkv, p, d = 1, 1, 32, 128
    geo = _geo(b, layers, hkv, p, d, "bf16")
    rng = np.random.default_rng(3)
    k, v = (torch.from_numpy(rng.standard_normal((1, 1, 1, p, d), dtype=np.float32)).bfloat16() for _ in range(2))
    k[0, 0, 0, 3, 40], v[0, 0, 0, 9, 17], v[0, 0, 0, 9, 18] = float("inf"), float("nan"), float("-inf")
    k[0, 0, 0, 5, 64:96] = 3.3e38
    pages = torch.zeros((1, b.packed_page_bytes(geo)), dtype=torch.uint8, device="cuda")
    packed = b.PackedPool(geo, pages)
    b.pack_pages(geo, b.PagePool(geo, k.cuda(), v.cuda()), packed, 0, 1, _t([0]), _t([0]))
    for off in (None, torch.tensor([[5, 0, 0]], dtype=torch.int32).cuda()):
        ko, vo = torch.zeros_like(k).cuda(), torch.zeros_like(v).cuda()
        b.unpack_rebase_pages(geo, packed, b.PagePool(geo, ko, vo), 0, 1, _t([0]), _t([0]), off)
        nk, nv = np.isnan(f64(ko))[0, 0, 0], np.isnan(f64(vo))[0, 0, 0]
        want = np.zeros((p, d), bool)
        want[3, 32:64] = True
        if off is not None:
            want[3, 96:128] = True
        assert (nk == want).all()
        want[:] = False
        want[:, 17:19] = True
        assert (nv == want).all()
    assert np.isfinite(f64(ko)[0, 0, 0, 5]).all()


def test_streams_graphs_and_large_offsets(b):
    """On a stream of its own, captured and replayed with other contents, pages behind 4 GiB."""
    layers, hkv, p, d = 36, 8, 256, 256
    geo = _geo(b, layers, hkv, p, d, "bf16")
    n = b.packed_page_bytes(geo)
    pages = torch.zeros((220, n), dtype=torch.uint8, device="cuda")  # 4.4 GB
    assert 219 * n > 2 ** 32
    pool = b.PagePool(geo, *(torch.randn((2, layers, hkv, p, d), device="cuda").bfloat16() for _ in range(2)))
    back = b.PagePool(geo, *(torch.zeros((2, layers, hkv, p, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    packed, src, dst, to = b.PackedPool(geo, pages), _t([1]), _t([219]), _t([0])
    stream = torch.cuda.Stream()

    def step():
        b.pack_pages(geo, pool, packed, 0, layers, src, dst)
        b.unpack_rebase_pages(geo, packed, back, 0, layers, dst, to)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(3):
        for t in pool.tensors:
            t.normal_()
        for t in back.tensors:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y, axis in zip(pool.tensors, back.tensors, (-1, -2)):
            x = x[1, 35, 7].double().cpu().numpy()
            c, s = op.blocks(np.ascontiguousarray(x if axis == -1 else x.T))
            want = op.value(c, np.repeat(s, 32, axis=-1))
            assert (f64(y[0, 35, 7]) == (want if axis == -1 else want.T)).all()
        assert not pages[:219].any()
