"""Every instance of the batch attention, chosen by the block tables' room and the max_rows hint, with room far from
the borders between them; and what a call may not touch, for batches of a plan and for arrays that no plan gives.

Which row tile (16, 32 or 64 query vectors) a call took is read from the workspace: where pieces are cut, the
statistics lie behind the outputs of 2 x 512 row tiles, and nothing behind those is written."""
import numpy as np
import pytest

from tests.batch_util import Case, ancestors, check_attend, tree

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

INSTANCES = [((6, 2, 32, "bf16"), 4), ((12, 1, 64, "bf16"), 4), ((6, 2, 96, "bf16"), 2), ((16, 2, 128, "bf16"), 2),
             ((2, 1, 256, "bf16"), 1), ((5, 5, 16, "f32"), 4), ((4, 1, 32, "f32"), 4), ((3, 1, 64, "f32"), 2),
             ((8, 2, 128, "f32"), 2)]  # geometry, the most groups of 16 query vectors in a row tile
ROOM = 8e9  # bytes; the borders lie between 24 and 240 MB
GUARD = 1 << 16


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _case(seed, geo, trees, cached=(900, 0, 90, 333), new=(17, 40, 1, 0), page=16, room=ROOM):
    rng = np.random.default_rng(seed)
    masks = sum([ancestors(tree(rng, n)) for n in new], []) if trees else None
    c = Case(seed, cached, new, page, *geo, masks=masks, pad_rows=2, layers=1)
    token = geo[1] * geo[2] * (2 if geo[3] == "bf16" else 4) * 2
    blocks = int(room / len(cached) / token / page) - c.max_blocks
    if blocks > 0:
        c.table = np.pad(c.table, ((0, 0), (0, blocks)), constant_values=-1)
        c.max_blocks += blocks
    return c


class Call:
    """One call with guards round what it writes; .check() looks at them and at what it reads."""

    def __init__(self, c, max_rows, narrow=False):
        from paper_2607_19547_amd import binding as b
        self.b, self.c = b, c
        self.geo, self.pool, self.batch, self.q, _, _ = c.dev(b, max_rows)
        self.size = b.tree_attend_paged_workspace(self.geo, self.batch)
        self.ws = torch.full((self.size + 2 * GUARD,), 255, dtype=torch.uint8, device="cuda")
        n, h, d = self.q.shape
        self.rows = torch.full((n + 8, h + 2, d + (2 if narrow else 0)), 7.0, dtype=self.q.dtype, device="cuda")
        self.out = self.rows[4:-4, 1:-1, (2 if narrow else 0):]  # narrow: aligned to two elements alone
        self.lses = torch.full((n + 8, h), 7.0, dtype=torch.float32, device="cuda")
        self.lse = self.lses[4:-4]
        self.reads = [x for x in self.batch.tensors if x is not None] + [self.q, *self.pool.tensors]

    def run(self):
        b = self.b
        before = [x.clone() for x in self.reads]
        b.cs_trace_reset()
        b.cs_trace_enable(True)
        b.tree_attend_paged(self.geo, self.pool, 0, self.batch, self.q, self.out, self.lse,
                            self.ws[GUARD:GUARD + self.size])
        torch.cuda.synchronize()
        b.cs_trace_enable(False)
        self.kernels = set(b.cs_trace_collect())
        b.cs_trace_reset()
        for x, y in zip(self.reads, before):  # (bits: NaN too)
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)), "an input changed"
        rest = self.rows.clone()
        rest[4:-4, 1:-1, -self.out.shape[2]:] = 7.0
        assert bool((rest == 7.0).all()) and bool((self.lses[:4] == 7.0).all()) and bool((self.lses[-4:] == 7.0).all())
        assert bool((self.ws[:GUARD] == 255).all()) and bool((self.ws[GUARD + self.size:] == 255).all())
        return self

    def groups(self, most):
        """The groups of 16 query vectors in the call's row tiles."""
        ws, d, found = self.ws[GUARD:GUARD + self.size], self.c.d, 0
        for g in (1, 2, 4):
            at = 2 * 512 * 16 * g * d * 4
            if g <= most and bool((ws[at:at + 2 * 512 * 16 * g * 8] != 255).any()):
                found = g
        return found


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("geo,most", INSTANCES)
def test_each_row_tile(geo, most, trees):
    """Row tiles of 16 (fetched once, by the hint), of 32 and of 64 query vectors; the requests have up to 40 rows."""
    g = geo[0] // geo[1]
    for seed, (groups, max_rows) in enumerate(((1, 1), (2, 240 // g), (4, 4000))):
        c = _case(seed, geo, trees)
        narrow = geo[2:] == (128, "bf16") and groups > 1  # else the kernel for many rows takes it
        call = Call(c, max_rows, narrow).run()
        what = f"{geo} max_rows {max_rows}"
        check_attend(c, 0, call.out, call.lse, what)
        assert "tree_attend" in call.kernels and call.kernels <= {"tree_attend", "tree_combine"}, (what, call.kernels)
        assert call.groups(most) == min(groups, most), what


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("geo,most", INSTANCES)
def test_little_room(geo, most, trees):
    """Row tiles of 16, fetched as usual."""
    c = _case(3, geo, trees, room=0)
    call = Call(c, 3).run()
    check_attend(c, 0, call.out, call.lse, str(geo))
    assert call.kernels <= {"tree_attend", "tree_combine"} and call.groups(most) == 1


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("max_rows", [8, 4000])
def test_many_rows(max_rows, trees):
    """The kernel for many rows, with the non-temporal hint (one row tile expected) and without."""
    c = _case(4, (16, 2, 128, "bf16"), trees)
    call = Call(c, max_rows).run()
    check_attend(c, 0, call.out, call.lse, f"max_rows {max_rows}")
    assert call.kernels == {"tree_attend_wide", "tree_combine_wide"}


@pytest.mark.parametrize("geo,most", INSTANCES)
def test_values_that_are_not_finite_in_every_row_tile(geo, most):
    """Row 1 of each request holds NaN and infinities that its descendants alone see."""
    for seed, max_rows in enumerate((1, 4000)):
        rng = np.random.default_rng(seed)
        new = (40, 33)
        masks = sum([ancestors([-1, -1] + [int(rng.integers(0, i)) for i in range(2, n)]) for n in new], [])
        c = _case(seed, geo, False, (37, 620), new)
        c.mask = masks
        for b in range(2):
            j = c.cached[b] + 1
            at = c.table[b][j // 16], slice(None), slice(None), j % 16
            c.v[at][..., 0], c.v[at][..., 1], c.v[at][..., 2] = float("inf"), float("-inf"), float("nan")
            if b:
                c.k[at] = float("nan")
        narrow = geo[2:] == (128, "bf16") and max_rows > 1
        call = Call(c, max_rows, narrow).run()
        check_attend(c, 0, call.out, call.lse, f"{geo} max_rows {max_rows}")
        assert call.groups(most) == (1 if max_rows == 1 else most)


PATHS = [((16, 2, 128, "bf16"), 1, ROOM), ((16, 2, 128, "bf16"), 4000, ROOM), ((12, 1, 64, "bf16"), 4000, ROOM),
         ((8, 2, 128, "f32"), 100, ROOM), ((5, 5, 16, "f32"), 4000, 0), ((2, 1, 80, "bf16"), 0, 0)]


@pytest.mark.parametrize("geo,max_rows,room", PATHS)
@pytest.mark.parametrize("start,cached", [([0, 4, 1 << 30], [20, 30]), ([0, 9, 3], [20, 30]), ([-5, 4, 8], [-3, 1 << 30]),
                                          ([0, 4, 8], [0x7fffffff, 30]), ([7, 2, 5], [20, -1 << 31]),
                                          ([0, 1 << 30, -1], [0x7fffffff, 0x7fffffff])])
def test_arrays_that_are_no_plans_touch_nothing_else(geo, max_rows, room, start, cached):
    """Row starts and lengths out of range: rows that no request owns keep what they hold, guards and inputs too."""
    c = _case(6, geo, False, (20, 30), (4, 4), room=room)
    call = Call(c, max_rows)
    call.batch.tensors[1].copy_(torch.tensor(start, dtype=torch.int32))
    call.batch.tensors[0].copy_(torch.tensor(cached, dtype=torch.int64).int())
    call.run()
    owned = np.zeros(c.n_rows, bool)
    for b in range(2):
        lo = min(max(start[b], 0), c.n_rows)
        owned[lo:max(min(start[b + 1], c.n_rows), lo)] = True
    rest = torch.from_numpy(~owned).cuda()
    assert bool((call.out[rest] == 7.0).all()) and bool((call.lse[rest] == 7.0).all())
