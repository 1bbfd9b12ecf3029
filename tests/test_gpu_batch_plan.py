"""batch_plan_pages and tree_commit_paged on the GPU against the oracle (whole numbers: equal)."""
import numpy as np
import pytest

from oracle import batch as ob
from tests.batch_util import rnd, tree

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _t(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def _geo(b, page, layers=1, hkv=1, d=16, dtype="f32"):
    return b.Geo(layers, hkv, hkv, d, (2, 3, 3) if d == 16 else (d // 2, 0, 0), dtype, [0, page])


class Step:
    """The arrays of one plan call; outputs hold a pattern before it."""

    def __init__(self, page, cached, new, held, table, free, head, n_rows, parent=None, base=None, words=1,
                 n_pages=1_000_000, mask=None):
        from paper_2607_19547_amd import binding as b
        n = len(cached)
        want_mask = parent is not None if mask is None else mask
        full = None if parent is None else list(parent) + [0] * (n_rows - len(parent))
        self.table, self.slot, self.coords = _t(table), _t(np.full(n_rows, 77)), _t(np.full((n_rows, 3), 77))
        self.row_start = _t(np.full(n + 1, 77))
        self.mask = _t(np.full((n_rows, words), 77), np.int64) if want_mask else None
        self.held_out, self.head_out, self.status = _t(np.full(n, 77)), _t([77]), _t([0])
        self.batch = b.Batch(_t(cached), self.row_start, self.table, self.slot, self.coords, self.mask)
        self.plan = b.PagePlan(_t(new), _t(held), self.held_out, _t(free), _t([head]), self.head_out, self.status,
                               parent=None if full is None else _t(full), coord_base=None if base is None else _t(base))
        self.geo, self.n_pages, self.call = _geo(b, page), n_pages, b.batch_plan_pages

    def run(self):
        self.call(self.geo, self.n_pages, self.batch, self.plan)
        torch.cuda.synchronize()
        return self


def _random(seed, n, page, most_cached, most_new, trees, words=1, pad_rows=0, base=True, zero=0.2):
    g = np.random.default_rng(seed)
    cached = np.where(g.random(n) < zero, 0, g.integers(0, most_cached + 1, n))
    new = np.where(g.random(n) < zero, 0, g.integers(0, most_new + 1, n))
    held = -(-cached // page) + g.integers(0, 3, n)  # some hold more pages than they fill
    need = np.maximum(held, -(-(cached + new) // page))
    width = int(need.max()) + 1
    grow = int((need - held).sum())
    order = g.permutation(int(held.sum()) + grow + 9)
    table = np.full((n, width), -7)
    at = 0
    for b in range(n):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.concatenate([[500, 501], order[at:]])
    rows = int(new.sum())
    parent = sum([tree(g, int(x)) for x in new], []) if trees else None
    args = dict(page=page, cached=cached, new=new, held=held, table=table, free=free, head=2, n_rows=rows + pad_rows,
                parent=parent, base=g.integers(-50, 100000, n) if base else None, words=words)
    return args


@pytest.mark.parametrize("kw", [
    dict(n=1, page=64, most_cached=9000, most_new=1, trees=False, zero=0.0),
    dict(n=1, page=1, most_cached=5, most_new=5, trees=True, zero=0.0),
    dict(n=3, page=16, most_cached=100, most_new=40, trees=True, pad_rows=5),
    dict(n=7, page=48, most_cached=1000, most_new=64, trees=True, pad_rows=300),
    dict(n=200, page=7, most_cached=50, most_new=20, trees=False, base=False),
    dict(n=257, page=64, most_cached=3000, most_new=64, trees=True),
    dict(n=5, page=33, most_cached=300, most_new=1500, trees=False, pad_rows=1),
    dict(n=4, page=64, most_cached=300, most_new=300, trees=True, words=5),
    dict(n=3, page=64, most_cached=30, most_new=2900, trees=True, words=46),  # trees longer than the LDS window
    dict(n=4096, page=16, most_cached=60, most_new=3, trees=True),
])
@pytest.mark.parametrize("seed", [0, 1])
def test_plan_equals_the_oracle(kw, seed):
    a = _random(seed, **kw)
    s = Step(**a).run()
    ref = ob.plan(**{k: v for k, v in a.items()})
    assert s.status.item() == 0
    assert s.row_start.tolist() == ref["row_start"] and s.table.tolist() == ref["table"]
    assert s.held_out.tolist() == ref["held"] and s.head_out.item() == ref["head"]
    assert s.slot.tolist() == ref["slot"]
    used = ref["row_start"][-1]
    assert s.coords[:used].tolist() == ref["coords"] and (s.coords[used:] == 77).all()
    if a["parent"] is not None and used:
        assert np.array_equal(s.mask[:used].cpu().numpy(), ob.mask_words(ref["mask"], a["words"]))
        assert (s.mask[used:] == 77).all()


def test_plan_writes_chain_masks_without_parents():
    a = _random(3, n=5, page=16, most_cached=40, most_new=130, trees=False, words=3)
    s = Step(**a, mask=True).run()
    ref = ob.plan(**a)
    assert np.array_equal(s.mask.cpu().numpy(), ob.mask_words(ref["mask"], 3))


def test_plan_of_no_rows():
    s = Step(16, [5, 0], [0, 0], [1, 0], [[4], [-1]], [3], 0, 0).run()
    assert s.row_start.tolist() == [0, 0, 0] and s.held_out.tolist() == [1, 0] and s.status.item() == 0


def test_plan_of_no_requests():
    s = Step(16, [], [], [], np.zeros((0, 4)), [3], 0, 4).run()
    assert s.row_start.tolist() == [0] and s.slot.tolist() == [-1] * 4 and s.head_out.item() == 0


@pytest.mark.parametrize("what,flag", [
    (dict(cached=[5, -1]), 1), (dict(new=[2, -3]), 1), (dict(held=[1, -1]), 1), (dict(held=[0, 2]), 1),
    (dict(cached=[5, 0x7fffffff], held=[1, 1]), 1), (dict(head=-1), 1),
    (dict(new=[2, 80], n_rows=90, words=2), 2), (dict(free=[7]), 4), (dict(head=9), 4), (dict(n_rows=10), 8),
    (dict(new=[2, 0x7fffffff]), 8), (dict(words=0), 16),
])
def test_a_step_that_cannot_be_planned_takes_nothing(what, flag):
    base = dict(page=16, cached=[5, 20], new=[2, 30], held=[1, 2], table=[[4, -1, -1, -1, -1], [2, 3, -1, -1, -1]],
                free=[7, 8, 9], head=0, n_rows=40)
    a = dict(base, **what)
    if "words" in what:  # a mask of one word, and a request of more than 64 rows
        a = dict(base, new=[2, 65], n_rows=90, mask=True, words=1, held=[1, 3]) if flag == 16 else dict(a, mask=True)
        if flag == 16:
            a["table"] = [[4] + [-1] * 7, [2, 3, 5] + [-1] * 5]
    s = Step(**a).run()
    assert s.status.item() & flag, s.status.item()
    assert s.table.tolist() == a["table"] and s.held_out.tolist() == a["held"] and s.head_out.item() == a["head"]
    assert s.row_start.tolist() == [0] * 3 and s.slot.tolist() == [-1] * a["n_rows"]
    assert (s.coords == 77).all()


def test_plan_flags_bad_parents_and_pages_and_keeps_earlier_flags():
    a = dict(page=16, cached=[5], new=[4], held=[1], table=[[4, -1]], free=[7], head=0, n_rows=4)
    s = Step(**a, parent=[-1, 1, 0, 9])
    s.status.fill_(64)
    s.run()
    assert s.status.item() == 32 + 64
    assert s.mask[:, 0].tolist() == [1, 2, 5, 8]  # a bad parent is the context
    a.update(cached=[15], held=[1], free=[2000], n_pages=1000)
    s = Step(**a).run()
    assert s.status.item() == 64 and s.slot.tolist() == [4 * 16 + 15, -1, -1, -1] and s.table.tolist() == [[4, 2000]]


def test_plan_captured_and_replayed_with_new_lengths():
    from paper_2607_19547_amd import binding as b
    cached, new, held = _t([5, 20, 0]), _t([3, 1, 0]), _t([1, 2, 0])
    table = _t(np.array([[4, -1, -1], [2, 3, -1], [-1] * 3]))
    rs, slot, coords = _t(np.zeros(4)), _t(np.zeros(8)), _t(np.zeros((8, 3)))
    ho, head, head_out, status, free = _t(np.zeros(3)), _t([0]), _t([0]), _t([0]), _t(np.arange(100, 120))
    batch = b.Batch(cached, rs, table, slot, coords)
    plan = b.PagePlan(new, held, ho, free, head, head_out, status)
    geo = _geo(b, 16)
    b.batch_plan_pages(geo, 1000, batch, plan)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.batch_plan_pages(geo, 1000, batch, plan)
    for step in range(4):
        c, n, h, t0 = cached.tolist(), new.tolist(), held.tolist(), table.tolist()
        want = ob.plan(16, c, n, h, t0, free.tolist(), head.item(), 8)
        g.replay()
        torch.cuda.synchronize()
        assert slot.tolist() == want["slot"] and table.tolist() == want["table"] and rs.tolist() == want["row_start"]
        cached.add_(new)
        held.copy_(ho)
        head.copy_(head_out)
        new.copy_(_t([step, 3, 2]))
    assert status.item() == 0


# ------------------------------------------------------------------ commit
@pytest.mark.parametrize("page,layers,hkv,d,dtype", [(16, 3, 2, 128, "bf16"), (7, 1, 1, 16, "f32"), (64, 36, 2, 128, "bf16"),
                                                     (5, 2, 3, 6, "bf16"), (1, 1, 2, 10, "f32")])
@pytest.mark.parametrize("seed", [0, 1])
def test_commit_equals_the_oracle(page, layers, hkv, d, dtype, seed):
    from paper_2607_19547_amd import binding as b
    g = np.random.default_rng(seed)
    n, most = 5, 80
    cached, new = g.integers(0, 90, n), g.integers(1, 110, n)
    need = -(-(cached + new) // page)
    order = g.permutation(int(need.sum()) + 3)
    table = np.full((n, int(need.max())), -1)
    at = 0
    for i in range(n):
        table[i, :need[i]] = order[at:at + need[i]]
        at += need[i]
    acc = np.full((n, most), -1)
    count = np.zeros(n, int)
    for i in range(n):
        count[i] = min(most, int(g.integers(0, new[i] + 1)))
        acc[i, :count[i]] = np.sort(g.choice(new[i], count[i], replace=False))
    count[0], acc[0] = most, np.arange(most)          # more than the request has rows, nothing to move
    acc[1, :4], count[1] = [0, 0, 1, 2], 4            # does not ascend
    count[2] = 1000                                   # beyond the list: what is -1 ends it
    kp, vp = (rnd(g, (len(order), layers, hkv, page, d), dtype) for _ in range(2))
    rs = np.concatenate([[0], np.cumsum(new)])
    geo = _geo(b, page, layers, hkv, d, dtype)
    pool = b.PagePool(geo, kp.cuda(), vp.cuda())
    rows = int(rs[-1])
    batch = b.Batch(_t(cached), _t(rs), _t(table), _t(np.zeros(rows)), _t(np.zeros((rows, 3))))
    out = _t(np.zeros(n))
    lb = layers // 3
    b.tree_commit_paged(geo, pool, lb, layers, batch, _t(acc), _t(count), out)
    rk, rv = kp.float().numpy().copy(), vp.float().numpy().copy()
    want = ob.commit([rk, rv], (lb, layers), cached, new, table.tolist(), acc.tolist(), count)
    assert out.tolist() == want
    assert np.array_equal(pool.tensors[0].float().cpu().numpy(), rk) and np.array_equal(pool.tensors[1].float().cpu().numpy(), rv)


def test_commit_leaves_out_bad_pages_and_empty_batches():
    from paper_2607_19547_amd import binding as b
    geo = _geo(b, 4)
    kp = torch.randn(3, 1, 1, 4, 16, device="cuda")
    pool = b.PagePool(geo, kp, kp.clone())
    before = kp.clone()
    table = _t([[0, 99], [-1, 1]])
    batch = b.Batch(_t([2, 2]), _t([0, 6, 12]), table, _t(np.zeros(12)), _t(np.zeros((12, 3))))
    out = _t([0, 0])
    b.tree_commit_paged(geo, pool, 0, 1, batch, _t([[1, 3], [2, 4]]), _t([2, 2]), out)
    # request 0: token 3 -> 2 in page 0; token 5 -> 3 has no page; request 1: nothing lies in the pool but page 1's rows
    want = before.clone()
    want[0, 0, 0, 2] = before[0, 0, 0, 3]
    assert torch.equal(pool.tensors[0], want) and out.tolist() == [4, 4]
    b.tree_commit_paged(geo, pool, 0, 0, batch, _t([[1, 3], [2, 4]]), _t([2, 2]), out)  # no layers: the lengths alone
    assert torch.equal(pool.tensors[0], want)
