"""tree_attend_paged on the GPU against the float64 oracle; tolerances in batch_util."""
import numpy as np
import pytest

from tests.batch_util import Case, ancestors, check_attend, f64, tree

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _run(c, layer=1, max_rows=0, ws=None, q=None, out=None, lse=True, stream=None, parts=None):
    from paper_2607_19547_amd import binding as b
    geo, pool, batch, q0, out0, lse0 = parts or c.dev(b, max_rows)
    if ws is None:
        ws = torch.empty(max(1, b.tree_attend_paged_workspace(geo, batch)), dtype=torch.uint8, device="cuda")
        ws.fill_(255)
    b.tree_attend_paged(geo, pool, layer, batch, q0 if q is None else q, out0 if out is None else out,
                        lse0 if lse else None, ws, stream=stream)
    torch.cuda.synchronize()
    return (out0 if out is None else out), lse0


def _check(c, layer=1, again=True, **kw):
    out, lse = _run(c, layer, **kw)
    check_attend(c, layer, out, lse, f"{c.cached} + {c.new}, page {c.page}, {c.hq}/{c.hkv} x {c.d} {c.dtype}")
    assert (out[c.rows:] == 7).all() and (lse[c.rows:] == 7).all(), "rows behind the last request changed"
    if again and c.d == 128 and c.dtype == "bf16":  # with the kernel for many rows too
        _check(c.roomy(), layer, again=False, **kw)


SHAPES = [  # cached, new, page
    ([0], [1], 16), ([1], [1], 16), ([31], [1], 64), ([32], [1], 32), ([300], [1], 48), ([1000], [1], 16),
    ([63, 0, 64, 65, 500], [1, 1, 1, 1, 1], 64), ([2000], [5], 128), ([129, 17], [3, 30], 16), ([0, 0], [70, 1], 32),
    ([77, 0, 400], [0, 0, 33], 48), ([40] * 9, [1, 2, 0, 4, 5, 6, 7, 8, 9], 7), ([513, 1], [130, 257], 64)]
GEOS = [(16, 2, 128, "bf16"), (5, 5, 128, "bf16"), (12, 1, 64, "bf16"), (6, 2, 96, "bf16"), (4, 2, 16, "f32"),
        (8, 2, 128, "f32"), (3, 1, 64, "f32"), (2, 1, 80, "bf16"), (4, 4, 10, "f32"), (2, 1, 256, "bf16"),
        (20, 1, 128, "bf16"), (2, 2, 32, "bf16"), (3, 3, 512, "f32")]


@pytest.mark.parametrize("geo", GEOS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_chains(geo, shape):
    cached, new, page = SHAPES[shape]
    _check(Case(shape, cached, new, page, *geo, pad_rows=shape % 3))


@pytest.mark.parametrize("geo", GEOS[:8])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_trees(geo, shape):
    cached, new, page = SHAPES[shape]
    rng = np.random.default_rng(shape)
    masks = sum([ancestors(tree(rng, n)) for n in new], [])
    _check(Case(shape, cached, new, page, *geo, masks=masks, pad_rows=shape % 2))


@pytest.mark.parametrize("geo", [GEOS[0], GEOS[2], GEOS[5], GEOS[7]])
def test_masks_that_leave_rows_empty(geo):
    """Any mask is allowed: none at all, later rows, bits of rows that the request does not have."""
    rng = np.random.default_rng(5)
    new, cached = [9, 40, 3, 70], [0, 0, 50, 0]
    masks = [0 if rng.random() < 0.4 else int(rng.integers(0, 1 << 62)) << int(rng.integers(0, 66)) for _ in range(sum(new))]
    masks[0], masks[9], masks[10] = 0, 1 << 39, 1 << 45
    masks = [m & (1 << 128) - 1 for m in masks]
    c = Case(5, cached, new, 16, *geo, masks=masks)
    _check(c)


@pytest.mark.parametrize("geo", [GEOS[0], GEOS[2], GEOS[5], GEOS[7]])
@pytest.mark.parametrize("new", [[3, 4], [40, 20]])
def test_infinities_and_nan_in_places_a_row_does_not_see(geo, new):
    """Rows 1 of each request holds NaN and infinities: only its descendants see them.  Pages' rows
    behind the last token and pages of nobody are NaN."""
    cached = [45, 2]
    rng = np.random.default_rng(1)
    masks = []
    for n in new:
        par = [-1, -1] + [int(rng.integers(0, 2)) if i < 4 else int(rng.integers(0, i)) for i in range(2, n)]
        masks += ancestors(par)
    c = Case(2, cached, new, 16, *geo, masks=masks)
    live = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
    for b in range(2):
        for j in range(cached[b] + new[b]):
            live[c.table[b][j // 16], j % 16] = True
    for x in (c.k, c.v):
        x.masked_fill_(~live[:, None, None, :, None], float("nan"))
    for b in range(2):
        j = cached[b] + 1
        c.v[c.table[b][j // 16], :, :, j % 16, 0] = float("inf")
        c.v[c.table[b][j // 16], :, :, j % 16, 1] = float("-inf")
        c.v[c.table[b][j // 16], :, :, j % 16, 2] = float("nan")
        if b:
            c.k[c.table[b][j // 16], :, :, j % 16] = float("nan")
    _check(c)
    c.mask = None  # a chain: row 0 alone does not see it
    _check(c)


def test_extreme_scores():
    """Scores that leave one key, a running maximum that keeps growing, and equal keys."""
    for seed, std in ((0, 60.0), (1, 0.0)):
        c = Case(seed, [700, 90], [3, 17], 32, 16, 2, 128, std_q=std)
        _check(c)
    c = Case(3, [600], [2], 32, 4, 2, 128)
    ramp = torch.linspace(0.0, 3.0, c.n_pages * 32).view(c.n_pages, 1, 1, 32, 1).to(c.k.dtype)
    order = torch.argsort(torch.from_numpy(c.table[0][:c.n_pages - 2]).long())
    full = torch.zeros_like(c.k)
    for x in range(c.n_pages - 2):
        full[c.table[0][x]] = ramp[x]
    c.k.copy_(full.abs())
    c.q.copy_(c.q.abs())
    assert len(order)
    _check(c)


def test_pages_outside_the_pool_are_not_seen():
    for geo in (GEOS[0], GEOS[5], GEOS[7]):
        c = Case(4, [200, 70], [2, 9], 32, *geo)
        c.table[0][1], c.table[0][3], c.table[1][0] = -1, c.n_pages, 1 << 30
        _check(c)


@pytest.mark.parametrize("geo,room", [(GEOS[0], False), (GEOS[0], True), (GEOS[5], False), (GEOS[7], False)])
def test_arrays_that_are_no_plans(geo, room):
    """Row starts and lengths out of range: bounded, nothing else is touched."""
    from paper_2607_19547_amd import binding as b
    c = Case(6, [20, 30], [4, 4], 16, *geo, pad_rows=2)
    if room:
        c.roomy()
    parts = c.dev(b)
    for start, cached in (([0, 4, 1 << 30], [20, 30]), ([0, 9, 3], [20, 30]), ([-5, 4, 8], [-3, 1 << 30]),
                          ([0, 4, 8], [0x7fffffff, 30])):
        parts[2].tensors[1].copy_(torch.tensor(start, dtype=torch.int32))
        parts[2].tensors[0].copy_(torch.tensor(cached, dtype=torch.int32))
        _run(c, parts=parts)


@pytest.mark.parametrize("geo", [GEOS[0], GEOS[5], GEOS[6]])
def test_strides_in_place_and_no_lse(geo):
    from paper_2607_19547_amd import binding as b
    c = Case(7, [333, 64], [6, 21], 48, *geo)
    parts = c.dev(b)
    want, _ = _run(c, parts=parts)
    want = want.clone()
    heads = parts[3].transpose(0, 1).contiguous().transpose(0, 1)  # [H][n][D]
    wide = torch.full((c.n_rows, c.hq + 3, c.d), 5.0, dtype=want.dtype, device="cuda")
    out, _ = _run(c, parts=parts, q=heads, out=wide[:, 1:1 + c.hq], lse=False)
    assert torch.equal(out, want) and (wide[:, 0] == 5).all() and (wide[:, -2:] == 5).all()
    two = torch.full((c.n_rows, c.hq * c.d + 2), 5.0, dtype=want.dtype, device="cuda")  # out aligned to two elements
    out, lse = _run(c, parts=parts, out=two[:, 2:].unflatten(1, (c.hq, c.d)))
    check_attend(c, 1, out, lse, "out aligned to two elements")
    assert (two[:, :2] == 5).all()
    own = parts[3].clone()
    out, _ = _run(c, parts=parts, q=own, out=own)  # in place, aligned
    assert torch.equal(out, want)
    odd = torch.zeros(c.n_rows, c.hq * c.d + 1, dtype=want.dtype, device="cuda")  # nothing aligned
    q = odd[:, 1:].unflatten(1, (c.hq, c.d))
    q.copy_(parts[3])
    out, lse = _run(c, parts=parts, q=q, out=q)
    check_attend(c, 1, out, lse, "unaligned, in place")


@pytest.mark.parametrize("max_rows", [1, 2, 8, 100, 4000])
def test_max_rows_is_a_hint(max_rows):
    """Any hint gives the results, for a batch of one-row and many-row requests."""
    _check(Case(8, [500, 70, 1500], [1, 90, 2], 64, 16, 2, 128), max_rows=max_rows)
    _check(Case(8, [500, 70], [1, 40], 48, 4, 2, 64, "f32"), max_rows=max_rows)


@pytest.mark.parametrize("geo", [GEOS[0], GEOS[2], GEOS[5]])
@pytest.mark.parametrize("new", [[1, 1], [1, 30]])
def test_block_tables_with_much_room(geo, new):
    """The room chooses how keys are fetched and how rows are tiled; the rest of a table is not read."""
    _check(Case(14, [700, 90], new, 64, *geo, pad_blocks=2000))


def test_short_batches_of_one_piece():
    for cached, new in (([0], [1]), ([3], [2]), ([100], [1])):
        for geo in ((2, 1, 128, "bf16"), (1, 1, 128, "f32"), (40, 1, 128, "bf16")):
            _check(Case(15, cached, new, 16, *geo, pad_blocks=0))


@pytest.mark.parametrize("geo", [GEOS[0], GEOS[1], GEOS[2], GEOS[4], GEOS[6]])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_units_shorter_than_a_run(geo, new):
    """Requests of a few keys each: a run has one of their units, or, where there are more than runs, some."""
    for seed, (n, cached) in enumerate(((2, 3), (40, 20), (9, 300))):
        lengths = np.random.default_rng(seed).integers(0, cached + 1, n).tolist()
        _check(Case(16, lengths, [(new * (b + 1)) % (new + 1) for b in range(n)], 16, *geo, layers=1, pad_rows=1), 0)


@pytest.mark.parametrize("geo,new", [((4, 2, 128, "bf16"), [720, 1, 613]), (GEOS[2], [400, 5, 530]), (GEOS[4], [500, 0, 600]), (GEOS[5], [300, 2, 313])])
def test_long_chains(geo, new):
    """Row tiles that see few and many keys, taken in pairs (where requests are many, some here without
    rows): with and without a cache, of odd and even numbers."""
    from paper_2607_19547_amd import binding as b
    c = Case(17, [0, 700, 333] + [0] * 37, new + [0] * 37, 64, *geo, layers=1, pad_rows=3).roomy()
    _check(c, 0, again=False)
    parts = c.dev(b)  # and lengths and a chain that a plan would not give
    for cached in (0x7fffffff, -5):
        parts[2].tensors[0].copy_(torch.tensor([cached, 700, cached] + [0] * 37, dtype=torch.int32))
        _run(c, 0, parts=parts)


def test_many_requests_and_a_long_one():
    rng = np.random.default_rng(9)
    cached = rng.integers(0, 40, 300).tolist()
    cached[17] = 9000
    _check(Case(9, cached, rng.integers(0, 3, 300).tolist(), 16, 4, 2, 128, layers=1), layer=0)


def test_long_cache_offsets_beyond_32_bits():
    """Pages more than 4 GiB from the pool's start."""
    from paper_2607_19547_amd import binding as b
    c = Case(10, [150], [3], 64, 16, 2, 128, layers=1)
    page_bytes = 2 * 64 * 128 * 2
    n_pages = (5 << 30) // page_bytes
    geo, pool, batch, q, out, lse = c.dev(b)
    big = [torch.zeros(n_pages, 1, 2, 64, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far = [n_pages - 1, n_pages - 7, n_pages // 2 + 5]
    for x, t in zip(big, (c.k, c.v)):
        for i, p in enumerate(far):
            x[p] = t[c.table[0][i]].cuda()
    batch.tensors[2][0, :3] = torch.tensor(far, dtype=torch.int32)
    pool = b.PagePool(geo, *big)
    out, lse = _run(c, 0, parts=(geo, pool, batch, q, out, lse))
    check_attend(c, 0, out, lse)


@pytest.mark.parametrize("geo,new,room", [(GEOS[0], [1, 1, 1], False), (GEOS[0], [40, 1, 20], False), (GEOS[0], [40, 1, 20], True),
                                          (GEOS[5], [3, 1, 20], False), (GEOS[7], [2, 1, 1], False)])
def test_same_bits_every_time_on_any_stream_and_replayed(geo, new, room):
    from paper_2607_19547_amd import binding as b
    c = Case(11, [3000, 100, 4500], new, 64, *geo)
    if room:
        c.roomy()
    parts = c.dev(b)
    geo, pool, batch, q, out, lse = parts
    want, want_lse = (x.clone() for x in _run(c, parts=parts))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, got_lse = _run(c, parts=parts)
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)
    ws = torch.empty(max(1, b.tree_attend_paged_workspace(geo, batch)), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.tree_attend_paged(geo, pool, 1, batch, q, out, lse, ws)
    lengths = batch.tensors[0]
    # (the third request's table has room for its own length alone, the second's for 100 tokens and a page)
    for cached in ([3000, 100, 4500], [5, 0, 64], [3000, 100, 4500], [1, 60, 17]):
        lengths.copy_(torch.tensor(cached, dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        eager, eager_lse = _run(c, parts=parts)
        assert torch.equal(got, eager) and torch.equal(got_lse, eager_lse)
        if cached[0] == 3000:
            assert torch.equal(got, want)


def test_two_calls_at_once_with_workspaces_of_their_own():
    from paper_2607_19547_amd import binding as b
    cases = [Case(s, [2500, 900], [n, n], 64, 16, 2, 128) for s, n in ((12, 1), (13, 40))]
    cases[1].roomy()
    parts = [c.dev(b) for c in cases]
    want = [[x.clone() for x in _run(c, parts=p)] for c, p in zip(cases, parts)]
    ws = [torch.empty(max(1, b.tree_attend_paged_workspace(p[0], p[2])), dtype=torch.uint8, device="cuda") for p in parts]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for p, w, s in zip(parts, ws, streams):
            b.tree_attend_paged(p[0], p[1], 1, p[2], p[3], p[4], p[5], w, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for p, w in zip(parts, want):
        assert torch.equal(p[4], w[0]) and torch.equal(p[5], w[1])


def test_binding_refuses_other_memory_types_and_geometries():
    from paper_2607_19547_amd import binding as b
    c = Case(16, [30], [2], 16, 4, 2, 128)
    geo, pool, batch, q, out, lse = c.dev(b)
    ws = torch.empty(b.tree_attend_paged_workspace(geo, batch), dtype=torch.uint8, device="cuda")
    call = lambda **kw: b.tree_attend_paged(kw.get("geo", geo), pool, 0, batch, kw.get("q", q), kw.get("out", out),
                                            kw.get("lse", lse), kw.get("ws", ws))
    call()
    other = b.Geo(2, 8, 4, 128, (16, 24, 24), "bf16", [0, 16])
    big = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(q=q.cpu()), dict(q=q.float()), dict(q=q[:, :2]), dict(q=q[:1]), dict(out=out.cpu()), dict(lse=lse.cpu()),
               dict(lse=lse.double()), dict(ws=ws.cpu()), dict(lse=lse[:1]), dict(geo=other, q=big, out=big, lse=None)):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(b.CsError) as e:
        call(ws=ws[:8])
    assert e.value.code == b.CS_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(ValueError):
        b.tree_commit_paged(geo, pool, 0, 2, batch, torch.zeros(1, 3, dtype=torch.int64, device="cuda"), batch.tensors[0])
    with pytest.raises(ValueError):
        b.Batch(*[t.cpu() if i == 2 else t for i, t in enumerate(batch.tensors[:5])])
