"""A memory packed page by page while it is answered from: pack, plan, norm and rotation, attention, commit and
restore together, over several steps of two requests that share packed pages.  Every call is checked against the
oracle on what the pages held before it; plan, append and attention of a step are also replayed from a graph."""
import numpy as np
import pytest

from oracle import batch as ob
from oracle import packed as op
from tests.batch_util import ancestors, f64, rnd, sections, theta, tree
from tests.packed_util import tol

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


def _t(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32")])
@pytest.mark.parametrize("sinks,window", [(0, 0), (6, 75)])
def test_answer_while_pages_are_packed(d, dtype, sinks, window):
    from paper_2607_19547_amd import binding as b
    rng = np.random.default_rng(d + window)
    L, hq, hkv, P, n_pages, n4, max_rows, eps = 2, 8, 2, 32, 40, 24, 16, 1e-6
    sec, th = sections(d), theta(d)
    page = b.Geo(L, hq, hkv, d, sec, dtype, [0, P])
    kp, vp = (rnd(rng, (n_pages, L, hkv, P, d), dtype).cuda() for _ in range(2))
    pool = b.PagePool(page, kp, vp)
    bits = torch.zeros((n4, b.packed_page_bytes(page)), dtype=torch.uint8, device="cuda")
    packed = b.PackedPool(page, bits)
    order, order4 = rng.permutation(n_pages), rng.permutation(n4)
    # a memory of six pages: four are packed at once; both requests see them, one goes on in pages of its own
    b.pack_pages(page, pool, packed, 0, L, _t(order[:4]), _t(order4[:4]))
    table = np.full((2, 20), -1)
    table[0, :6] = np.concatenate([order4[:4], order[4:6]])
    table[1, :4] = order4[:4]
    table = _t(table)
    cached, held, blocks = _t([6 * P - 9, 4 * P]), _t([6, 4]), _t([4, 4])
    held_out, head, head_out, status = _t([0, 0]), _t([0]), _t([0]), _t([0])
    free = _t(order[6:])  # (the packed pages' places in the pool could be handed out again)
    arrays = dict(row_start=_t([0, 0, 0]), slot=_t(np.zeros(max_rows)), coords=_t(np.zeros((max_rows, 3))),
                  mask=_t(np.zeros((max_rows, 1)), np.int64))
    new, parent, base = _t([0, 0]), _t(np.zeros(max_rows)), _t([300, 200])
    batch = b.Batch(cached, arrays["row_start"], table, arrays["slot"], arrays["coords"], arrays["mask"])
    plan = b.PagePlan(new, held, held_out, free, head, head_out, status, parent=parent, coord_base=base)
    ws = torch.empty(b.tree_attend_packed_workspace(page, batch), dtype=torch.uint8, device="cuda")
    wk = rnd(rng, (d,), dtype).cuda().add_(1.0)
    x = rnd(rng, (max_rows, hq + 2 * hkv, d), dtype, 1.5).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    q_out = torch.zeros((max_rows, hq, d), dtype=kp.dtype, device="cuda")
    out, lse = torch.zeros_like(q_out), torch.zeros(max_rows, hq, device="cuda")
    cached_out = _t([0, 0])
    layer, next4 = 1, 4

    def step():
        b.batch_plan_pages(page, n_pages, batch, plan)
        b.qk_norm_rope_append(page, pool, layer, batch, q, k, v, q_out, None, wk, eps)
        b.tree_attend_packed(page, pool, packed, layer, batch, blocks, q_out, out, lse, ws, sinks=sinks, window=window)

    graph = None
    for lengths in ([7, 5], [1, 1], [9, 7], [3, 0], [1, 15], [8, 8]):
        drafted = lengths[0] in (9, 1)
        par = [tree(rng, n) if drafted else list(range(-1, n - 1)) for n in lengths]
        flat = sum(par, [])
        new.copy_(_t(lengths))
        parent.copy_(_t(flat + [0] * (max_rows - len(flat))))
        x.copy_(rnd(rng, tuple(x.shape), dtype, 1.5))
        c = cached.tolist()
        want = ob.plan(P, c, lengths, held.tolist(), table.tolist(), free.tolist(), head.item(), max_rows, flat,
                       base.tolist())
        bits_before = bits.clone()
        if graph is None:
            step()
            torch.cuda.synchronize()
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                step()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
            torch.cuda.synchronize()
        else:
            graph.replay()
        assert status.item() == 0 and table.tolist() == want["table"] and held_out.tolist() == want["held"]
        assert torch.equal(bits, bits_before), "a step writes packed pages"
        rows = sum(lengths)
        ref, ref_lse, spread = np.zeros((rows, hq, d)), np.zeros((rows, hq)), np.zeros((rows, hq, d + 2))
        k4, v4 = op.decode(bits.cpu().numpy(), L, hkv, P, d)
        masks = [m for p in par for m in ancestors(p)]
        op.attend(f64(q_out), f64(kp), f64(vp), k4, v4, layer, c, want["row_start"], want["table"], blocks.tolist(), masks,
                  sinks, window, ref, ref_lse, spread)
        t_out, t_lse = tol(ref, ref_lse, spread, dtype)
        assert (np.abs(f64(out[:rows]) - ref) <= t_out).all() and (np.abs(f64(lse[:rows]) - ref_lse) <= t_lse).all()
        # accept a path, then pack the pages that are full by now
        acc = np.full((2, 16), -1)
        for i, p in enumerate(par):
            j, path = len(p) - 1, []
            while j >= 0:
                path.append(j)
                j = p[j]
            acc[i, :len(path)] = path[::-1]
        count = (acc >= 0).sum(1)
        b.tree_commit_paged(page, pool, 0, L, batch, _t(acc), _t(count), cached_out)
        assert torch.equal(bits, bits_before), "a commit writes packed pages"
        cached.copy_(cached_out)
        held.copy_(held_out)
        head.copy_(head_out)
        base.add_(_t(count))
        for r in range(2):
            done = blocks.tolist()[r]
            full = cached.tolist()[r] // P
            if full > done:
                n = full - done
                src, dst = table[r, done:full].clone(), _t(order4[next4:next4 + n])
                b.pack_pages(page, pool, packed, 0, L, src, dst)
                table[r, done:full] = dst
                blocks[r] = full
                got = bits[dst.long()].cpu().numpy()
                assert (got == op.encode(f64(kp)[src.tolist()], f64(vp)[src.tolist()])).all()
                next4 += n
    assert next4 >= 6, "fewer than two pages were packed on the way"
    # the memory moves back into the pool, elsewhere on the timeline
    n = blocks.tolist()[0]
    ko, vo = torch.zeros_like(kp), torch.zeros_like(vp)
    off = np.repeat([[11, -2, 3]], n, axis=0)
    b.unpack_rebase_pages(page, packed, b.PagePool(page, ko, vo), 0, L, table[0, :n].contiguous(), _t(np.arange(n)), _t(off))
    k4, v4 = (a[table[0, :n].tolist()] for a in op.decode(bits.cpu().numpy(), L, hkv, P, d))
    ang = off[0][np.repeat(np.arange(3), sec)] * th
    u, w = k4[..., :d // 2], k4[..., d // 2:]
    turned = np.concatenate([u * np.cos(ang) - w * np.sin(ang), u * np.sin(ang) + w * np.cos(ang)], -1)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    pair = np.concatenate([np.hypot(u, w)] * 2, -1)
    assert (np.abs(f64(ko)[:n] - turned) <= pair * 6 * 2.0 ** -24 + half * np.abs(turned) * 1.01).all()
    assert (f64(vo)[:n] == v4).all()
