"""A memory composed in pages by the paged calls, then answered from: plan,
norm and rotation, attention and commit together, over several steps of two
requests that share pages.  Every call is checked against the oracle on what
the pages held before it."""
import numpy as np
import pytest

from oracle import batch as ob
from tests.batch_util import attend_tol, f64, rnd, sections, theta, tree
from tests.gpu_util import pair_norm

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _t(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def _compose(b, geo, k, v, fresh, offsets):
    """Re-base, select and repair a composed cache held as chunk tensors; returns the selection."""
    n = geo.g.n_tokens - 64 * 2
    q, kf, vf = fresh
    b.compose_rebase_k_paged(geo, k, offsets)
    scores = torch.empty(n, dtype=torch.float32, device="cuda")
    sel = torch.empty(n, dtype=torch.int32, device="cuda")
    m = b.score_deviation_topk_paged(geo, k, 1, kf[1], 0.25, scores, sel)
    out = torch.empty((2, geo.g.n_q_heads, m, 128), dtype=q.dtype, device="cuda")
    ws = torch.empty(max(1, b.selective_attend_scatter_workspace(geo, m, 2)), dtype=torch.uint8, device="cuda")
    b.selective_attend_scatter_paged(geo, k, v, 0, 2, sel, m, q, kf, vf, out, None, ws)
    return sel[:m]


def test_compose_in_pages_then_answer():
    from paper_2607_19547_amd import binding as b
    rng = np.random.default_rng(0)
    L, hq, hkv, d, P, n_pages, eps = 2, 16, 2, 128, 64, 24, 1e-6
    sec, th = sections(d), theta(d)
    page = b.Geo(L, hq, hkv, d, sec, "bf16", [0, P])
    kp, vp = (rnd(rng, (n_pages, L, hkv, P, d), "bf16").cuda() for _ in range(2))
    pool = b.PagePool(page, kp, vp)
    order = rng.permutation(n_pages)
    mem = [int(x) for x in order[:6]]  # three chunks of two pages; the pages are used where they lie
    # the two pages of the first chunk are one request's whole memory and the start of the other's
    geo = b.Geo(L, hq, hkv, d, sec, "bf16", np.array([0, 128, 192, 256, 320, 384]))
    offsets = np.array([[0, 0, 0], [8, 0, 1], [8, 0, 1], [17, 0, 0], [17, 0, 0]])
    fresh = [rnd(rng, (L, h, 256, d), "bf16").cuda() for h in (hq, hkv, hkv)]

    # the same composition in buffers of its own
    first = [torch.cat([x[mem[0]], x[mem[1]]], dim=2).contiguous() for x in (kp, vp)]
    own = [[first[i]] + [x[p].clone() for p in mem[2:]] for i, x in enumerate((kp, vp))]
    sel_own = _compose(b, geo, own[0], own[1], fresh, offsets)
    # in the pool: the first chunk (offset zero, never written) as a tensor beside it, the others in their pages
    k_in, v_in = ([first[i].clone()] + [x[p] for p in mem[2:]] for i, x in enumerate((kp, vp)))
    sel = _compose(b, geo, k_in, v_in, fresh, offsets)
    assert torch.equal(sel, sel_own)
    for i, x in enumerate((kp, vp)):
        for j, p in enumerate(mem[2:]):
            assert torch.equal(x[p], own[i][1 + j]), "a page composed in the pool differs"

    # two requests: one over all six pages, 380 of 384 tokens; one over the first two, 128 tokens
    cached = _t([380, 128])
    table = _t(np.full((2, 12), -1))
    table[0, :6] = _t(mem)
    table[1, :2] = _t(mem[:2])
    held, held_out, head, head_out, status = _t([6, 2]), _t([0, 0]), _t([0]), _t([0]), _t([0])
    free = _t(order[6:])
    base = _t([400, 150])
    max_rows = 24
    arrays = dict(row_start=_t([0, 0, 0]), slot=_t(np.zeros(max_rows)), coords=_t(np.zeros((max_rows, 3))),
                  mask=_t(np.zeros((max_rows, 1)), np.int64))
    new, parent = _t([0, 0]), _t(np.zeros(max_rows))
    batch = b.Batch(cached, arrays["row_start"], table, arrays["slot"], arrays["coords"], arrays["mask"])
    plan = b.PagePlan(new, held, held_out, free, head, head_out, status, parent=parent, coord_base=base)
    ws = torch.empty(b.tree_attend_paged_workspace(page, batch), dtype=torch.uint8, device="cuda")
    wq, wk = (rnd(rng, (d,), "bf16").cuda().add_(1.0) for _ in range(2))
    out, lse = torch.zeros(max_rows, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(max_rows, hq, device="cuda")
    cached_out = _t([0, 0])

    for step, lengths in enumerate(([7, 5], [13, 9], [1, 1], [3, 0])):
        drafted = step == 1
        par = [tree(rng, n) if drafted else list(range(-1, n - 1)) for n in lengths]
        flat = sum(par, [])
        new.copy_(_t(lengths))
        parent.copy_(_t(flat + [0] * (max_rows - len(flat))))
        c, h, t0 = cached.tolist(), held.tolist(), table.tolist()
        want = ob.plan(P, c, lengths, h, t0, free.tolist(), head.item(), max_rows, flat, base.tolist())
        b.batch_plan_pages(page, n_pages, batch, plan)
        assert status.item() == 0
        assert table.tolist() == want["table"] and arrays["slot"].tolist() == want["slot"]
        assert held_out.tolist() == want["held"] and arrays["row_start"].tolist() == want["row_start"]
        rows = sum(lengths)
        assert arrays["coords"][:rows].tolist() == want["coords"]
        for layer in range(L):
            x = rnd(rng, (max_rows, hq + 2 * hkv, d), "bf16", 1.5).cuda()
            q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
            rk = ob.norm_rope(f64(k[:rows]), f64(wk), eps, want["coords"], sec, th)
            rq = ob.norm_rope(f64(q[:rows]), f64(wq), eps, want["coords"], sec, th)
            before = kp.clone()
            rv = f64(v[:rows])
            b.qk_norm_rope_append(page, pool, layer, batch, q, k, v, q, wq, wk, eps)  # queries in place
            slots = np.array(want["slot"][:rows])
            pg, off = slots // P, slots % P
            for got, ref in ((f64(q[:rows]), rq), (f64(kp)[pg, layer, :, off], rk)):
                tol = (d + 16) * 2.0 ** -24 * pair_norm(ref) * 1.01 + 2.0 ** -8 * np.abs(ref)
                assert (np.abs(got - ref) <= tol).all()
            assert np.array_equal(f64(vp)[pg, layer, :, off], rv)
            touched = torch.zeros(n_pages, P, dtype=torch.bool)
            touched[torch.from_numpy(pg), torch.from_numpy(off)] = True
            same = (kp == before)[:, layer].all(dim=3).all(dim=1).cpu()
            assert bool((same | touched).all()) and torch.equal(kp[:, 1 - layer], before[:, 1 - layer])
            b.tree_attend_paged(page, pool, layer, batch, q, out, lse, ws)
            ref, ref_lse, spread = np.zeros((rows, hq, d)), np.zeros((rows, hq)), np.zeros((rows, hq, d + 2))
            ob.attend(f64(q), f64(kp), f64(vp), layer, c, want["row_start"], want["table"], want["mask"], ref, ref_lse,
                      spread)
            t_out, t_lse = attend_tol(ref, ref_lse, spread, "bf16")
            assert (np.abs(f64(out[:rows]) - ref) <= t_out).all() and (np.abs(f64(lse[:rows]) - ref_lse) <= t_lse).all()
        # accept: a question's rows all, of a tree the way to its last node
        acc = np.full((2, 13), -1)
        for i, p in enumerate(par):
            j, path = len(p) - 1, []
            while j >= 0:
                path.append(j)
                j = p[j]
            acc[i, :len(path)] = path[::-1]
        count = (acc >= 0).sum(1)
        rk, rv = f64(kp), f64(vp)
        moved = ob.commit([rk, rv], (0, L), c, lengths, want["table"], acc, count)
        b.tree_commit_paged(page, pool, 0, L, batch, _t(acc), _t(count), cached_out)
        assert cached_out.tolist() == moved and np.array_equal(f64(kp), rk) and np.array_equal(f64(vp), rv)
        cached.copy_(cached_out)
        held.copy_(held_out)
        head.copy_(head_out)
        base.add_(_t(count))
