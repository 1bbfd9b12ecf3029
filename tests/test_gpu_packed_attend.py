"""Attention over packed pages and over windows against float64, element by element."""
import numpy as np
import pytest

from tests.batch_util import ancestors, f64, tree
from tests.packed_util import PackedCase, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FAST = [(16, 2, 128, "bf16"), (5, 5, 128, "bf16"), (12, 1, 64, "bf16"), (6, 2, 96, "bf16"), (2, 1, 256, "bf16"),
        (2, 2, 32, "bf16"), (8, 2, 128, "f32"), (3, 1, 64, "f32"), (4, 1, 32, "f32")]
ANY = [(2, 1, 160, "bf16"), (4, 2, 224, "f32")]
SPAN_ONLY = [(4, 2, 16, "f32"), (2, 1, 80, "bf16")]  # no packed pages: D is no multiple of 32
MAIN = [FAST[0], FAST[2], FAST[6], ANY[0]]


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.fixture(scope="module")
def b(built_lib):
    from paper_2607_19547_amd import binding
    return binding


def _masks(rng, new, width=3):
    return [m for n in new for m in ancestors(tree(rng, n, width))]


@pytest.mark.parametrize("geo", FAST + ANY)
@pytest.mark.parametrize("page", [32, 96])
def test_one_token(b, geo, page):
    """A row each, lengths from none to many pages; all packed, none packed, some."""
    packed = [0, 1, 3, 0, 2, 7]
    cached = [0, page, 3 * page + 5, 45, 2 * page + 31, 7 * page + page - 1]
    check(PackedCase(1, packed, cached, [1] * 6, page, *geo), b)


@pytest.mark.parametrize("geo", FAST)
def test_one_token_in_tables_with_room(b, geo):
    """Tables that would hold much more: two packed tiles a step, of which the second may be none."""
    packed = [0, 1, 3, 17, 2, 40]
    c = PackedCase(20, packed, [9, 32, 100, 17 * 32 + 31, 95, 40 * 32], [1] * 6, 32, *geo)
    blocks = int(50e3 / 6 / geo[1]) + 1
    c.table = np.pad(c.table, ((0, 0), (0, blocks)), constant_values=-1)
    c.max_blocks += blocks
    check(c, b)
    c.sinks, c.window = 40, 2 ** 30
    check(c, b)


@pytest.mark.parametrize("geo", FAST + ANY)
@pytest.mark.parametrize("masked", [False, True])
def test_several_rows(b, geo, masked):
    rng = np.random.default_rng(5)
    new = [7, 1, 19, 0, 3]
    c = PackedCase(2, [5, 0, 2, 1, 3], [5 * 64 + 3, 0, 150, 64, 3 * 64], new, 64, *geo,
                   masks=_masks(rng, new) if masked else None, pad_rows=2)
    check(c, b)


@pytest.mark.parametrize("geo", [FAST[0], FAST[2], FAST[6], FAST[7]])
@pytest.mark.parametrize("new", [[70], [33, 90]])
def test_many_rows(b, geo, new):
    """Row tiles of more than 16 query vectors, several of them."""
    c = PackedCase(3, [9] * len(new), [9 * 32 + 11] * len(new), new, 32, *geo, layers=1)
    check(c, b, 0)


@pytest.mark.parametrize("geo", FAST + ANY + SPAN_ONLY)
@pytest.mark.parametrize("sinks,window", [(0, 1), (4, 40), (37, 64), (3, 700), (500, 500), (2 ** 31 - 1, 1), (0, 2 ** 31 - 1)])
def test_windows(b, geo, sinks, window):
    """Sinks and windows that end inside tiles, meet, reach beyond everything; single tokens and chains."""
    span_only = geo in SPAN_ONLY
    page = 16 if span_only else 32
    packed = None if span_only else [20, 0, 5, 1]
    cached, new = [700, 90, 32 * 5, 40], [1, 5, 40, 2]
    check(PackedCase(4, packed, cached, new, page, *geo, sinks=sinks, window=window), b)


@pytest.mark.parametrize("geo", MAIN)
@pytest.mark.parametrize("sinks,window", [(0, 2), (3, 1), (40, 5), (45, 9), (33, 300), (1, 64)])
def test_windows_of_trees(b, geo, sinks, window):
    """The window counts what a row sees: its ancestors, not its siblings.  Windows shorter than the tree is deep,
    sinks among the step's own rows, masks of two words."""
    rng = np.random.default_rng(sinks + window)
    new = [9, 80, 30, 66]
    cached = [0, 40, 32 * 9, 3]
    c = PackedCase(5, [0, 1, 9, 0], cached, new, 32, *geo, sinks=sinks, window=window, masks=_masks(rng, new, 2))
    check(c, b)


@pytest.mark.parametrize("geo", MAIN)
def test_arbitrary_masks(b, geo):
    """Masks that are no tree: rows that see nothing at all, later rows, bits behind the request's rows."""
    rng = np.random.default_rng(8)
    new = [6, 5]
    masks = [int(x) for x in rng.integers(0, 64, 6)] + [int(x) for x in rng.integers(0, 32, 5)]
    masks[0] = 0
    masks[6] = 0b11111
    for sinks, window, cached in ((0, 0, [0, 37]), (2, 2, [0, 37]), (1, 3, [64, 0])):
        c = PackedCase(9, [x // 32 for x in cached], cached, new, 32, *geo, sinks=sinks, window=window, masks=masks)
        check(c, b)


@pytest.mark.parametrize("geo", MAIN)
def test_windows_of_rows_without_rows(b, geo):
    """A row whose mask is empty sees `window` cached tokens, one more than a row that sees itself: the first of them may
    be the last of a tile that the other rows' windows leave out."""
    for packed, cached, window, sinks in (([2, 3], [95, 127], 32, 0), ([0, 5], [31 + 640, 63 + 640], 64, 5)):
        c = PackedCase(23, packed, cached, [2, 3], 32, *geo, sinks=sinks, window=window, masks=[0, 0b10, 0b111, 0, 0b100])
        check(c, b)


def test_clip_behind_ordinary_pages(b):
    """Many rows with a window and no packed page; pages of 16 and 48 tokens."""
    for geo in (FAST[0], FAST[2], FAST[7]):
        for page in (16, 48):
            check(PackedCase(6, None, [500, 0], [150, 90], page, *geo, sinks=4, window=100, layers=1), b, 0)


@pytest.mark.parametrize("geo", [FAST[0], FAST[6], FAST[2]])
def test_long(b, geo):
    """Many runs and their merge."""
    for window in (0, 5000):
        check(PackedCase(7, [400, 31], [400 * 32 + 9, 31 * 32 + 31], [1, 2], 32, *geo, layers=1, sinks=70, window=window), b, 0)


@pytest.mark.parametrize("geo", FAST)
def test_pages_outside_the_pools(b, geo):
    """Table entries of neither pool are not seen; an entry is of the pool that its place says."""
    c = PackedCase(10, [6, 2], [6 * 32 + 40, 64 + 9], [2, 1], 32, *geo, spare=1)
    c.table[0, 1], c.table[0, 4], c.table[1, 0], c.table[0, 6] = -1, c.n4, 2 ** 31 - 1, c.n_pages
    check(c, b)
    c.window, c.sinks = 50, 33
    check(c, b)


@pytest.mark.parametrize("geo", MAIN)
def test_counts_that_are_no_plan(b, geo):
    """packed_blocks beyond the cached tokens or below zero: whole pages of cached tokens count."""
    c = PackedCase(11, [3, 1, 2], [3 * 32 + 5, 40, 64], [2, 1, 1], 32, *geo)
    want = c.run(b)
    c.packed = [3, 1, 1000]
    got = c.run(b)
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    check(c, b)
    c.packed = [0, 0, -5]
    c.table[:] = c.table.clip(max=c.n_pages - 1)
    got = c.run(b)
    c.packed = [0, 0, 0]
    for x, y in zip(c.run(b), got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("geo", FAST + [ANY[0]])
@pytest.mark.parametrize("sinks,window", [(0, 0), (5, 70)])
def test_nan_blocks(b, geo, sinks, window):
    """A NaN block of a key makes the scores of its token NaN, one of the values an element of the output; rows that
    see none of its tokens are as without it."""
    from oracle import packed as op
    hq, hkv, d, dtype = geo
    p, new = 32, [30, 1]
    for seed, part in ((12, "v"), (13, "k"), (14, "both")):
        c = PackedCase(seed, [8, 3], [8 * 32 + 7, 3 * 32 + 1], new, p, *geo, sinks=sinks, window=window)
        n, s = p * d // 2, p * d // 32
        x = c.bits.reshape(c.n4, c.layers * hkv, -1)
        plane = 1 * hkv  # layer 1, head 0
        for blk in (1, 6, 7):  # hidden from some rows, or all, where there is a window
            pg = c.table[0, blk]
            if part in ("v", "both"):
                x[pg, plane, 2 * n + s + (5 if blk == 1 else d - 1)] = 255
            if part == "k" or part == "both" and blk == 1:
                x[pg, plane, n + 32 * (d // 32 - 1) + (9 if blk == 6 else 30)] = 255
        check(c, b, what=part)


@pytest.mark.parametrize("geo", [FAST[0], FAST[2], FAST[6], ANY[0]])
def test_values_that_are_not_finite_behind_windows(b, geo):
    """Infinities and NaN in ordinary pages: hidden by the window they do not matter, seen they do."""
    c = PackedCase(15, None, [200, 64], [4, 1], 32, *geo, sinks=3, window=60)
    for j in (3, 50, 143):
        c.k[c.table[0, j // 32], :, :, j % 32] = float("nan")
        c.v[c.table[0, j // 32], :, :, j % 32] = float("inf")
    check(c, b)
    c.v[c.table[0, 5], :, 0, 20, 7] = float("-inf")  # token 180: seen by every row
    check(c, b)


@pytest.mark.parametrize("geo", [FAST[0], FAST[6], FAST[5]])
def test_large_and_small_scales(b, geo):
    """Scales of both ends: scores far apart, outputs of 1e30 and of 1e-30."""
    from oracle import packed as op
    hq, hkv, d, dtype = geo
    for vs in (127 + 95, 127 - 100):
        c = PackedCase(16, [12], [12 * 32 + 3], [3], 32, *geo)
        n, s = 16 * d, d
        x = c.bits.reshape(c.n4, c.layers * hkv, -1)
        x[..., 2 * n + s:] = vs
        x[:, :, n:n + s] = c.rng.integers(2, 129, (c.n4, c.layers * hkv, s))
        c.v *= 2.0 ** (vs - 127)
        check(c, b)


@pytest.mark.parametrize("geo", [FAST[0], FAST[4], FAST[8], ANY[1]])
def test_strides_in_place_and_no_lse(b, geo):
    """Queries as slices of a projection's rows, outputs into one, out in place of q, unaligned rows, no lse."""
    hq, hkv, d, dtype = geo
    c = PackedCase(17, [4, 1], [4 * 32 + 9, 50], [5, 2], 32, *geo, window=90, sinks=2)
    want = c.run(b)[0]
    dt = want.dtype
    for pad in (8, 1):
        fused = torch.zeros((c.n_rows, hq * d + pad + 16), dtype=dt, device="cuda")
        q = fused[:, pad:pad + hq * d].unflatten(1, (hq, d))
        q.copy_(c.q)
        wide = torch.full((c.n_rows, hq, d + pad + 7), 3.0, dtype=dt, device="cuda")
        out = wide[:, :, pad:pad + d]
        got = c.run(b, q=q, out=out, lse=False)[0]
        ref, ref_lse, spread = c.attend_ref(1)
        from tests.packed_util import tol
        assert (np.abs(f64(got) - ref) <= tol(ref, ref_lse, spread, dtype)[0]).all()
        assert (wide[:, :, :pad] == 3).all() and (wide[:, :, pad + d:] == 3).all()
    q = c.q.cuda()
    assert torch.equal(c.run(b, q=q, out=q)[0], want)


@pytest.mark.parametrize("geo", [FAST[0], FAST[2]])
def test_same_as_without_packing(b, geo):
    """Without packed pages and window the call is tree_attend_paged; with all tokens seen a window changes nothing
    but, by rounding, the last bits."""
    c = PackedCase(18, None, [300, 20], [3, 1], 32, *geo)
    g, pool, batch, q, out, lse = c.dev(b)
    ws = torch.empty(b.tree_attend_paged_workspace(g, batch), dtype=torch.uint8, device="cuda")
    b.tree_attend_paged(g, pool, 1, batch, q, out, lse, ws)
    got = c.run(b)
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    c.window = 4000
    check(c, b)


def test_replays_and_two_streams(b):
    """Captured and replayed with other lengths; two calls at once with a workspace each."""
    c = PackedCase(19, [20, 3, 0], [20 * 32 + 5, 3 * 32 + 30, 70], [3, 1, 2], 32, *FAST[0], window=500, sinks=33)
    geo, pool, batch, q, out, lse = c.dev(b)
    packed = b.PackedPool(geo, torch.from_numpy(c.bits).cuda())
    blocks = torch.tensor(c.packed, dtype=torch.int32).cuda()
    ws = torch.empty(b.tree_attend_packed_workspace(geo, batch), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.tree_attend_packed(geo, pool, packed, 1, batch, blocks, q, out, lse, ws, sinks=33, window=500)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b.tree_attend_packed(geo, pool, packed, 1, batch, blocks, q, out, lse, ws, sinks=33, window=500)
    torch.cuda.synchronize()
    for cached, n in ((c.cached, c.packed), ([19 * 32 + 1, 70, 0], [19, 2, 0]), (c.cached, [4, 3, 0]), (c.cached, c.packed)):
        batch.tensors[0].copy_(torch.tensor(cached, dtype=torch.int32))
        blocks.copy_(torch.tensor(n, dtype=torch.int32))
        table = torch.from_numpy(c.table).cuda() % min(c.n4, c.n_pages)  # (each entry lies in both pools)
        batch.tensors[2].copy_(table)
        want, want_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
        ws2 = torch.empty_like(ws)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.tree_attend_packed(geo, pool, packed, 1, batch, blocks, q, want, want_lse, ws2, sinks=33, window=500)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("geo", [FAST[0], ANY[0]])
def test_pages_behind_four_gib(b, geo):
    """Packed pages far into a large pool, in the last of many layers."""
    from tests.packed_util import tol
    hq, hkv, d, dtype = geo
    layers = 36 if d == 128 else 24
    c = PackedCase(21, [5, 1], [5 * 32 + 9, 40], [2, 1], 32, *geo, layers=layers, sinks=33, window=70)
    g, pool, batch, q, out, lse = c.dev(b)
    n = 2 ** 32 // b.packed_page_bytes(g) + c.n4 + 1
    pages = torch.zeros((n, b.packed_page_bytes(g)), dtype=torch.uint8, device="cuda")
    pages[n - c.n4:] = torch.from_numpy(c.bits).cuda()
    table = batch.tensors[2]
    for r, k in enumerate(c.packed):
        table[r, :k] += n - c.n4
    ws = torch.empty(b.tree_attend_packed_workspace(g, batch), dtype=torch.uint8, device="cuda")
    ref, ref_lse, spread = c.attend_ref(layers - 1)
    blocks = torch.tensor(c.packed, dtype=torch.int32).cuda()
    for hint in (0, 2_000_000):
        batch.c.max_rows = hint
        out.fill_(7.0)
        b.tree_attend_packed(g, pool, b.PackedPool(g, pages), layers - 1, batch, blocks, q, out, lse, ws, sinks=33, window=70)
        assert (np.abs(f64(out) - ref) <= tol(ref, ref_lse, spread, dtype)[0]).all()


@pytest.mark.parametrize("geo", MAIN)
def test_runs_repeat_bit_by_bit(b, geo):
    """The same call again, with another workspace's contents, gives the same bits."""
    c = PackedCase(22, [60, 9, 0], [60 * 32 + 3, 300, 77], [3, 1, 2], 32, *geo, sinks=5, window=1500)
    first = c.run(b)
    again = c.run(b)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("sinks,window", [(0, 0), (7, 40)])
def test_full_batch(b, sinks, window):
    """4,096 requests, most of them over the same packed pages."""
    from tests.packed_util import tol
    rng = np.random.default_rng(24)
    n = 4096
    packed = [int(x) for x in rng.integers(0, 4, n)]
    cached = [32 * p + int(x) for p, x in zip(packed, rng.integers(0, 20, n))]
    c = PackedCase(25, [0] * n, [1] * n, [1] * n, 32, 2, 1, 32, sinks=sinks, window=window, layers=1)
    c.packed, c.cached = packed, cached
    from tests.packed_util import random_packed
    c.n4 = 5
    c.bits = random_packed(rng, 5, 1, 1, 32, 32)
    own = c.table[:, 0].copy()
    c.max_blocks = 6
    c.table = np.full((n, 6), -1, np.int32)
    for r in range(n):
        c.table[r, :packed[r]] = rng.permutation(5)[:packed[r]]
        c.table[r, packed[r]] = own[r]
    check(c, b, 0)


def test_refused_tensors(b):
    """What the binding itself refuses, before the library is called."""
    c = PackedCase(26, [1, 0], [40, 9], [1, 2], 32, *FAST[0])
    geo, pool, batch, q, out, lse = c.dev(b)
    bits = torch.from_numpy(c.bits).cuda()
    packed, blocks = b.PackedPool(geo, bits), torch.tensor(c.packed, dtype=torch.int32).cuda()
    ws = torch.empty(b.tree_attend_packed_workspace(geo, batch), dtype=torch.uint8, device="cuda")
    other = b.Geo(3, 16, 2, 128, (16, 24, 24), "bf16", [0, 32])
    for bad in (bits[:, 1:], bits[:, ::2], bits.to(torch.int32), bits.cpu()):
        with pytest.raises(ValueError):
            b.PackedPool(geo, bad)
    call = lambda **kw: b.tree_attend_packed(*[{**dict(geo=geo, pool=pool, packed=packed, layer=1, batch=batch, blocks=blocks,
                                                       q=q, out=out, lse=lse, ws=ws), **kw}[k]
                                               for k in ("geo", "pool", "packed", "layer", "batch", "blocks", "q", "out",
                                                         "lse", "ws")])
    for kw in (dict(packed=None), dict(geo=other), dict(blocks=blocks[:1]), dict(blocks=blocks.long()), dict(q=q[:2]),
               dict(q=q.float()), dict(out=out[:, :3]), dict(lse=lse[:2]), dict(lse=lse.double()), dict(ws=ws.cpu())):
        with pytest.raises(ValueError):
            call(**kw)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    for args in ((i32(0), i32(0, 1)), (i32(0).long(), i32(0)), (i32(0), i32(0).cpu())):
        with pytest.raises(ValueError):
            b.pack_pages(geo, pool, packed, 0, 1, *args)
        with pytest.raises(ValueError):
            b.unpack_rebase_pages(geo, packed, pool, 0, 1, *args)
    with pytest.raises(ValueError):
        b.unpack_rebase_pages(geo, packed, pool, 0, 1, i32(0), i32(0), i32(1, 2, 3))
    with pytest.raises(ValueError):
        b.pack_pages(other, pool, packed, 0, 1, i32(0), i32(0))
    call()
    torch.cuda.synchronize()
