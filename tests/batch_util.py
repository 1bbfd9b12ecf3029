"""Random batches over a pool of pages for the tests of the batch calls, and
the tolerances their outputs are held to."""
import numpy as np


def theta(d, base=1.0e6):
    return base ** (-2.0 * np.arange(d // 2) / d)


def sections(d):
    p = d // 2
    s = p // 4
    return s, (p - s) // 2, p - s - (p - s) // 2


def rnd(rng, shape, dtype, std=1.0):
    """A CPU tensor of normal draws in the storage type."""
    import torch
    x = torch.from_numpy(rng.standard_normal(shape, dtype=np.float32) * np.float32(std))
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def f64(t):
    return t.detach().cpu().double().numpy()


def tree(rng, n, width=3):
    """Parents of a random tree of n rows (several roots where it is wide)."""
    return [-1 if i == 0 or rng.random() < 0.1 else int(rng.integers(max(0, i - width), i)) for i in range(n)]


def ancestors(parent):
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


class Case:
    """A batch with its pages appended already: numpy/CPU side, `dev()` puts it on the GPU."""

    def __init__(self, seed, cached, new, page, hq, hkv, d, dtype="bf16", layers=2, masks=None, spare=2, pad_rows=0,
                 pad_blocks=1, std_q=1.5):
        from oracle import batch as ob
        self.rng = rng = np.random.default_rng(seed)
        self.cached, self.new, self.page, self.hq, self.hkv, self.d, self.dtype, self.layers = (
            list(cached), list(new), page, hq, hkv, d, dtype, layers)
        need = [-(-(c + n) // page) for c, n in zip(cached, new)]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.max_blocks = max(need, default=0) + pad_blocks
        self.table = np.full((len(need), self.max_blocks), -1, np.int32)
        at = 0
        for b, x in enumerate(need):
            self.table[b, :x] = order[at:at + x]
            at += x
        self.row_start = [0] + [int(x) for x in np.cumsum(new)]
        self.rows = self.row_start[-1]
        self.n_rows = self.rows + pad_rows
        self.k = rnd(rng, (self.n_pages, layers, hkv, page, d), dtype)
        self.v = rnd(rng, (self.n_pages, layers, hkv, page, d), dtype)
        self.q = rnd(rng, (self.n_rows, hq, d), dtype, std_q)
        self.mask = masks  # python ints per row, or None
        self.words = max(1, -(-max(new, default=1) // 64))
        self.ob = ob

    def roomy(self):
        """The same batch with block tables of so much room that several rows take the kernel for many."""
        blocks = int(120e6) // (max(len(self.new), 1) * self.page * self.hkv * self.d * 4) + 1
        self.table = np.pad(self.table, ((0, 0), (0, blocks)), constant_values=-1)
        self.max_blocks += blocks
        return self

    def geo(self, b):
        return b.Geo(self.layers, self.hq, self.hkv, self.d, sections(self.d), self.dtype, [0, self.page])

    def dev(self, b, max_rows=0):
        """(geo, pool, batch, q, out, lse) on the GPU; out and lse hold a pattern."""
        import torch
        t = lambda x: torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()
        geo = self.geo(b)
        slot = np.full(self.n_rows, -1, np.int32)
        m = None
        if self.mask is not None:
            m = np.full((self.n_rows, self.words), -1, np.int64)
            m[:self.rows] = self.ob.mask_words(self.mask, self.words)
            m = torch.from_numpy(m).cuda()
        batch = b.Batch(t(self.cached), t(self.row_start), t(self.table).reshape(len(self.cached), self.max_blocks),
                        t(slot), t(np.zeros((self.n_rows, 3))), m, max_rows=max_rows)
        pool = b.PagePool(geo, self.k.cuda(), self.v.cuda())
        q = self.q.cuda()
        out = torch.full_like(q, 7.0)
        lse = torch.full((self.n_rows, self.hq), 7.0, dtype=torch.float32, device="cuda")
        return geo, pool, batch, q, out, lse

    def attend_ref(self, layer):
        out = np.full((self.n_rows, self.hq, self.d), 7.0)
        lse = np.full((self.n_rows, self.hq), 7.0)
        spread = np.zeros((self.n_rows, self.hq, self.d + 2))
        self.ob.attend(f64(self.q), f64(self.k), f64(self.v), layer, self.cached, self.row_start, self.table.tolist(),
                       self.mask, out, lse, spread)
        return out, lse, spread


def attend_tol(out, lse, spread, dtype):
    """Bounds of |out - exact| and |lse - exact|, element by element.

    A score is a sum of D float32 products (bf16 products are exact), in any
    order: off by at most D 2^-24 of sum |q K| / sqrt(D), plus its scaling, the
    argument of the exponential in units of log2 and the exponential itself
    (16 such steps cover them); a running sum of n terms by n 2^-24.  That is the relative
    error of every p and of their sum, twice in the output.  In bf16 a p is
    also rounded once (2^-8 of it, so 2^-8 of sum p |V|), and the output is
    rounded once to its type."""
    d = out.shape[-1]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    s_abs, n = spread[..., d], spread[..., d + 1]
    rel = (d + 16) * 2.0 ** -24 * (1 + s_abs) + (n + 64) * 2.0 ** -24
    tol = spread[..., :d] * (2 * rel + (2.0 ** -8 if dtype == "bf16" else 0.0))[..., None]
    with np.errstate(invalid="ignore"):
        return tol * (1 + half) + half * np.abs(out) + 1e-30, rel + 2.0 ** -23 * np.abs(np.where(np.isfinite(lse), lse, 0))


def check_attend(case, layer, out, lse, what=""):
    ref, ref_lse, spread = case.attend_ref(layer)
    got, got_lse = f64(out), f64(lse)
    t_out, t_lse = attend_tol(ref, ref_lse, spread, case.dtype)
    assert (np.isnan(got) == np.isnan(ref)).all(), f"{what}: NaN where none belongs, or the other way round"
    fin = np.isfinite(ref)
    assert (got[~fin & ~np.isnan(ref)] == ref[~fin & ~np.isnan(ref)]).all(), f"{what}: infinities differ"
    bad = np.abs(got[fin] - ref[fin]) > t_out[fin]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outputs off by up to {np.abs(got[fin] - ref[fin]).max():.3e}"
    fin = np.isfinite(ref_lse)
    assert (np.isnan(got_lse) == np.isnan(ref_lse)).all() and (
        got_lse[~fin & ~np.isnan(ref_lse)] == ref_lse[~fin & ~np.isnan(ref_lse)]).all(), f"{what}: lse not finite"
    d = np.abs(got_lse[fin] - ref_lse[fin])
    assert (d <= t_lse[fin]).all(), f"{what}: lse off by up to {d.max(initial=0):.3e}"
