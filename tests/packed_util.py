"""Random batches whose first pages are packed, and the tolerances of attention over them."""
import numpy as np

from tests.batch_util import Case, attend_tol, f64


def random_packed(rng, n, layers, hkv, p, d):
    """Packed pages of random codes; scales from 2^-3 to 2^1, as normal draws have them."""
    s, c = p * d // 32, p * d // 2
    x = rng.integers(0, 256, (n, layers * hkv, 2 * (s + c)), dtype=np.uint8)
    for a in (c, 2 * c + s):
        x[:, :, a:a + s] = rng.integers(124, 129, (n, layers * hkv, s), dtype=np.uint8)
    return x.reshape(n, -1)


class PackedCase(Case):
    """A Case whose requests have `packed` [B] pages in a packed pool; sinks and window of the call."""

    def __init__(self, seed, packed, cached, new, page, hq, hkv, d, dtype="bf16", sinks=0, window=0, **kw):
        super().__init__(seed, cached, new, page, hq, hkv, d, dtype, **kw)
        from oracle import packed as op
        self.op, self.packed, self.sinks, self.window = op, packed, sinks, window
        self.n4 = (sum(packed) if packed else 0) + 2
        if packed is not None:
            self.bits = random_packed(self.rng, self.n4, self.layers, hkv, page, d)
            order, at = self.rng.permutation(self.n4), 0
            for b, n in enumerate(packed):
                self.table[b, :n] = order[at:at + n]
                at += n

    def run(self, b, layer=1, lse=True, out=None, q=None, ws=None, max_rows=0):
        import torch
        geo, pool, batch, dq, dout, dlse = self.dev(b, max_rows=max_rows)
        p4 = blocks = None
        if self.packed is not None:
            p4 = b.PackedPool(geo, torch.from_numpy(self.bits).cuda())
            blocks = torch.tensor(self.packed, dtype=torch.int32).cuda()
        if ws is None:
            ws = torch.empty(max(1, b.tree_attend_packed_workspace(geo, batch)), dtype=torch.uint8, device="cuda")
            ws.fill_(0xff)
        dout = dout if out is None else out
        b.tree_attend_packed(geo, pool, p4, layer, batch, blocks, dq if q is None else q, dout, dlse if lse else None, ws,
                             sinks=self.sinks, window=self.window)
        torch.cuda.synchronize()
        return dout, dlse

    def attend_ref(self, layer):
        out = np.full((self.n_rows, self.hq, self.d), 7.0)
        lse = np.full((self.n_rows, self.hq), 7.0)
        spread = np.zeros((self.n_rows, self.hq, self.d + 2))
        k4 = v4 = np.zeros((0,) + tuple(self.k.shape[1:]))
        if self.packed is not None:
            k4, v4 = self.op.decode(self.bits, self.layers, self.hkv, self.page, self.d)
        self.op.attend(f64(self.q), f64(self.k), f64(self.v), k4, v4, layer, self.cached, self.row_start,
                       self.table.tolist(), self.packed, self.mask, self.sinks, self.window, out, lse, spread)
        return out, lse, spread


def tol(out, lse, spread, dtype):
    """attend_tol's bounds; in float32 a score and an output are sums of three times as many products (three bf16
    terms of a query or a probability, each product exact), so three times the terms of those sums."""
    d = out.shape[-1]
    if dtype == "bf16":
        t, t_lse = attend_tol(out, lse, spread, dtype)
        if d == 128:
            # Many rows leave their pieces in fp16, scaled so that a row's largest element lies in [2^14, 2^15): half a
            # step is 2^-11 of an element, and at most 2^-25 where elements are so small that steps are even, which is
            # 2^-39 of the largest.  Weighted like the pieces' outputs, these add up to as much of sum p |V|.
            t = t + 2.0 ** -11 * spread[..., :d] + 2.0 ** -39 * spread[..., :d].max(-1, keepdims=True)
        return t, t_lse
    rel = (3 * d + 16) * 2.0 ** -24 * (1 + spread[..., d]) + (3 * spread[..., d + 1] + 64) * 2.0 ** -24
    with np.errstate(invalid="ignore"):
        t = spread[..., :d] * (2 * rel)[..., None] * (1 + 2.0 ** -24) + 2.0 ** -24 * np.abs(out) + 1e-30
        return t, rel + 2.0 ** -23 * np.abs(np.where(np.isfinite(lse), lse, 0))


def row_hints(case):
    """Values of max_rows that make the call take its other kernels: with the most rows the largest row tiles (or, in
    bf16 with heads of 128, the kernel for many rows), with fewer others."""
    keys = case.max_blocks * case.page
    if case.window:
        keys = min(keys, case.sinks + case.window + 32)
    tiles = max(1.0, len(case.cached) * keys * case.hkv / 32)
    def rows(work):
        return int(work / tiles * 16 / (case.hq // case.hkv)) + 1
    # row tiles of 16 and two tiles a step, row tiles of 32, of 64
    return sorted({0, rows(50e3), rows(200e3), 2_000_000})


def check(case, b, layer=1, what="", **kw):
    ref = case.attend_ref(layer)
    for hint in row_hints(case):
        out, lse = _check(case, b, layer, f"{what} max_rows {hint}", ref, max_rows=hint, **kw)
    return out, lse


def _check(case, b, layer, what, ref, **kw):
    out, lse = (f64(x) for x in case.run(b, layer, **kw))
    ref, ref_lse, spread = ref
    t_out, t_lse = tol(ref, ref_lse, spread, case.dtype)
    what = f"{what} packed {case.packed} cached {case.cached} new {case.new} {case.hq}/{case.hkv} x {case.d} " \
           f"{case.dtype} sinks {case.sinks} window {case.window}"
    assert (np.isnan(lse) == np.isnan(ref_lse)).all(), f"{what}: NaN lost or made in lse"
    assert (np.isnan(out) == np.isnan(ref)).all(), f"{what}: NaN lost or made ({np.isnan(out).sum()}, {np.isnan(ref).sum()})"
    fin = np.isfinite(ref)
    assert (out[~fin & ~np.isnan(ref)] == ref[~fin & ~np.isnan(ref)]).all(), f"{what}: infinities"
    bad = np.abs(out[fin] - ref[fin]) > t_out[fin]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off by up to {np.abs(out[fin] - ref[fin]).max():.3e}"
    ok = np.isfinite(ref_lse)
    assert (lse[~ok & ~np.isnan(ref_lse)] == ref_lse[~ok & ~np.isnan(ref_lse)]).all(), f"{what}: lse not finite"
    assert (np.abs(lse[ok] - ref_lse[ok]) <= t_lse[ok]).all(), f"{what}: lse off by {np.abs(lse[ok] - ref_lse[ok]).max():.3e}"
    return out, lse
