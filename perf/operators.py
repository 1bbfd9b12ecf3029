"""The operators that answer over a composed cache, as measurable cases.

A composed memory lives in pages, each a chunk buffer [L][H_kv][P][D] of the
paged calls; requests reach it through block tables.  One step of a batch of
requests is four operations (`op`):

  plan     block tables, slots, coordinates and tree masks of the step, built
           on the GPU from the requests' lengths
  append   per-head RMS norm and three-axis rotation of the step's queries and
           keys; keys and values go to their slots
  attend   attention of the step's rows over their requests' pages: a single
           token, a tree of drafted tokens, or the tokens of a question
  commit   the rows of an accepted path move behind the cached ones

A case is a dict of plain values.  `prepare` makes on the GPU what a user's
program holds before the call, `run` is one pass: elementary torch operations
where `own` is false, the package's entry points where it is true.  `exact` is
the same result in float64, from the operations' definitions.

Geometry is Qwen2.5-VL-3B's (16 query / 2 KV heads, head dim 128, sections
16/24/24, base 1e6) in bf16 unless a case says otherwise.
"""
import math

import numpy as np
import torch

own = False

BASE = 1.0e6
EPS = 1.0e-6
QWEN = dict(q_heads=16, kv_heads=2, dim=128, dtype="bf16")


def _case(op, **kw):
    c = dict(op=op, requests=1, cached=1024, new=1, tree=False, page=64, layers=2, ragged=False)
    c.update(QWEN)
    c.update(kw)
    return c


def listed():
    return [
        # The next token of one answer: the smallest plan there is.
        dict(_case("plan", requests=1, cached=8211, new=1), name="plan-1"),
        # A full server, every request with a tree of drafted tokens.
        dict(_case("plan", requests=512, cached=16384, new=64, tree=True, ragged=True), name="plan-512-trees"),
        # The next token's query, key and value: latency.
        dict(_case("append", new=1, cached=8211), name="append-1"),
        # Full-precision fidelity runs: a question of 1,999 tokens in float32.
        dict(_case("append", requests=3, new=1999, ragged=True, cached=1021, dtype="f32", page=48), name="append-2k-f32"),
        # The frames of one more clip, prefilled behind the memory (queries,
        # keys and values are slices of one projection's rows).
        dict(_case("append", requests=2, new=16381, cached=8192, page=128), name="append-32k"),
        # One answer's next token over a short video's memory.
        dict(_case("attend", cached=8211, new=1), name="decode-8k"),
        # A batch of answers over memories of very different lengths.
        dict(_case("attend", requests=32, cached=16384, new=1, ragged=True), name="decode-32"),
        # A tree of drafted tokens over a long video's memory.
        dict(_case("attend", cached=65501, new=61, tree=True, page=128), name="tree-65k"),
        # Float32: a few small trees over short memories.
        dict(_case("attend", requests=4, cached=4096, new=17, tree=True, ragged=True, dtype="f32", page=48),
             name="tree-4k-f32"),
        # Two questions of a few hundred tokens over long memories: the most
        # arithmetic of all.
        dict(_case("attend", requests=2, cached=32768, new=389, page=64), name="question-32k"),
        # One request's accepted path, all 36 layers.
        dict(_case("commit", cached=8211, new=61, tree=True, layers=36), name="commit-1"),
        # A batch's accepted paths, all 36 layers.
        dict(_case("commit", requests=48, cached=1500, new=64, tree=True, layers=36, ragged=True, page=32),
             name="commit-48"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(16, 2), (16, 2), (28, 4), (40, 8), (10, 10), (12, 1), (4, 2)]


def draw(rng):
    op = rng.choice(["plan", "append", "attend", "attend", "attend", "commit"])
    hq, hkv = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([128, 128, 128, 64]) if dtype == "bf16" else rng.choice([128, 64, 16])
    page = rng.choice([16, 32, 48, 64, 64, 128, 256])
    kw = dict(q_heads=hq, kv_heads=hkv, dim=dim, dtype=dtype, page=page, ragged=rng.random() < 0.7)
    per_token = hkv * dim * (2 if dtype == "bf16" else 4) * 2  # bytes of a token's K and V in a layer
    if op == "plan":
        tree = rng.random() < 0.6
        requests = _log_int(rng, 1, 512)
        new = _log_int(rng, 1, 64 if tree else max(1, 32768 // requests))
        return _case(op, **dict(kw, requests=requests, cached=_log_int(rng, 1, 16384), new=new, tree=tree))
    if op == "append":
        rows = _log_int(rng, 1, max(2, 30000 * (18 * 128 * 2) // ((hq + hkv) * dim * (2 if dtype == "bf16" else 4))))
        requests = min(rows, _log_int(rng, 1, 64))
        return _case(op, **dict(kw, requests=requests, cached=_log_int(rng, 1, 4096), new=max(1, rows // requests)))
    if op == "commit":
        requests = _log_int(rng, 1, 48)
        layers = rng.choice([4, 12, 28, 36])
        cached = _log_int(rng, 1, max(1, min(1500, 2_000_000_000 // (per_token * layers * requests) - 128)))
        return _case(op, **dict(kw, requests=requests, cached=cached, new=_log_int(rng, 2, 64), tree=True,
                                layers=layers))
    shape = rng.choice(["decode", "tree", "question"])
    requests = _log_int(rng, 1, 64)
    most = max(2, 262144 * 1024 // per_token // requests)  # tokens a request's memory may have at most
    cached = _log_int(rng, 1, min(65536, most))
    if shape == "decode":
        return _case(op, **dict(kw, requests=requests, cached=cached, new=1))
    # rows so that the products stay below the largest listed case's
    # (float32: a sixteenth of it, by the rates of the matrix instructions)
    budget = 2 * 389 * 16 * 128 * 33000 // (1 if dtype == "bf16" else 16)
    rows = max(1, budget // (requests * hq * dim * (cached + 256)))
    if shape == "tree":
        return _case(op, **dict(kw, requests=requests, cached=cached, new=min(rows, _log_int(rng, 2, 128)), tree=True))
    return _case(op, **dict(kw, requests=requests, cached=cached, new=min(rows, _log_int(rng, 2, 512))))


# ------------------------------------------------------------------ a batch's sizes
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _sections(c):
    p = c["dim"] // 2
    s = p // 4
    return s, (p - s) // 2, p - s - (p - s) // 2


def _lengths(c):
    """(cached, new) of every request; they depend on the case alone, so that a
    case's work does not vary with the seed.  Ragged: spread from a sixteenth of
    the case's length to all of it."""
    g = np.random.Generator(np.random.PCG64(c["requests"] * 1000003 + c["cached"] * 101 + c["new"]))
    cached = np.full(c["requests"], c["cached"], dtype=np.int64)
    new = np.full(c["requests"], c["new"], dtype=np.int64)
    if c["ragged"]:
        cached = np.maximum(1, np.exp(g.uniform(math.log(max(1.0, c["cached"] / 16)), math.log(c["cached"] + 0.5),
                                                c["requests"])).astype(np.int64))
        cached[0] = c["cached"]
        if c["new"] > 1:
            new = np.maximum(1, g.integers((c["new"] + 1) // 2, c["new"] + 1, c["requests"]))
            new[0] = c["new"]
    return cached, new


def _mask_words(c):
    return max(1, -(-c["new"] // 64))


def _parents(c, new, g):
    """Trees in breadth-first order: node 0 hangs on the context, eight
    alternatives follow it, and each level's nodes hang on random ones of the
    level before."""
    out = []
    for n in new:
        par, prev = [-1], [0]
        while len(par) < n:
            level = list(range(len(par), min(int(n), len(par) + 8)))
            par += [int(prev[int(g.integers(0, len(prev)))]) for _ in level]
            prev = level
        out += par
    return np.asarray(out, dtype=np.int32)


def _path(parent):
    """An accepted path: the way from the root to the last node, cut off where
    the rows it moves to would reach a row it moves from, so that a pass can be
    made again on the same state."""
    i, path = len(parent) - 1, []
    while i >= 0:
        path.append(i)
        i = int(parent[i])
    path = path[::-1]
    while any(j != i and j < len(path) for i, j in enumerate(path)):
        path.pop()
    return path


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _normal(shape, gen, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    return x.normal_(0.0, std, generator=gen)


# ------------------------------------------------------------------ prepare
def prepare(case, seed):
    c = dict(case)
    g = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    cached, new = _lengths(c)
    B, P, H, D, L = c["requests"], c["page"], c["kv_heads"], c["dim"], c["layers"]
    rows = int(new.sum())
    need = -(-(cached + new) // P)
    held = -(-cached // P)
    width = int(need.max()) + 3
    n_pages = int(need.sum()) + 5
    order = g.permutation(n_pages).astype(np.int32)
    st = dict(c=c, n_pages=n_pages, n_rows=rows, layer=L - 1, theta=_theta(c))
    # the block table: the pages held before the step, or with the step's own
    have = held if c["op"] == "plan" else need
    table = np.full((B, width), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
    row_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    req = np.repeat(np.arange(B), new)
    idx = np.arange(rows) - row_start[req]
    parent = _parents(c, new, g) if c["tree"] else None
    st.update(cached_len=_dev(cached.astype(np.int32)), table=_dev(table))
    words = _mask_words(c)
    if c["op"] == "plan":
        st.update(new_len=_dev(new.astype(np.int32)), n_blocks=_dev(held.astype(np.int32)), free=_dev(order[at:]),
                  free_head=_dev(np.array([2], dtype=np.int32)),
                  coord_base=_dev(g.integers(0, 100_000, B).astype(np.int32)),
                  parent=None if parent is None else _dev(parent))
        for name, shape, t in (("row_start", (B + 1,), torch.int32), ("slot", (rows,), torch.int32),
                               ("coords", (rows, 3), torch.int32), ("n_blocks_out", (B,), torch.int32),
                               ("free_head_out", (1,), torch.int32)):
            st[name] = torch.empty(shape, dtype=t, device="cuda")
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")  # flags are added to it
        st["mask"] = torch.empty((rows, words), dtype=torch.int64, device="cuda") if c["tree"] else None
    else:
        pos = cached[req] + idx
        slot = table[req, pos // P].astype(np.int64) * P + pos % P
        st.update(row_start=_dev(row_start), slot=_dev(slot.astype(np.int32)), mask=None)
        coords = np.repeat((g.integers(0, 100_000, B)[req] + idx)[:, None], 3, axis=1)
        if c["op"] == "append":  # image tokens: three different coordinates
            coords = coords + np.stack([np.zeros(rows, np.int64), g.integers(0, 32, rows), g.integers(0, 32, rows)], 1)
        st["coords"] = _dev(coords.astype(np.int32))
        if c["op"] == "attend" and c["tree"]:
            bits = np.zeros((rows, words), dtype=np.uint64)
            for r in range(rows):
                i = int(idx[r])
                p = int(parent[r])
                if p >= 0:
                    bits[r] = bits[r - i + p]
                bits[r, i // 64] |= np.uint64(1) << np.uint64(i % 64)
            st["mask"] = _dev(bits.view(np.int64))
        dt = _dtype(c)
        st["kp"] = _normal((n_pages, L, H, P, D), gen, dt)
        st["vp"] = _normal((n_pages, L, H, P, D), gen, dt)
        if c["op"] == "append":
            fused = _normal((rows, (c["q_heads"] + 2 * H) * D), gen, dt, 1.7).view(rows, -1, D)
            st["q"], st["k"], st["v"] = (fused[:, :c["q_heads"]], fused[:, c["q_heads"]:c["q_heads"] + H],
                                         fused[:, c["q_heads"] + H:])
            st["wq"], st["wk"] = (_normal((D,), gen, torch.float32, 0.2).add_(1.0).to(dt) for _ in range(2))
            st["q_out"] = torch.empty((rows, c["q_heads"], D), dtype=dt, device="cuda")
        elif c["op"] == "attend":
            st["q"] = _normal((rows, c["q_heads"], D), gen, dt, 1.5)
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((rows, c["q_heads"]), dtype=torch.float32, device="cuda")
        else:
            paths = [_path(parent[row_start[b]:row_start[b + 1]]) for b in range(B)]
            most = max(len(p) for p in paths)
            acc = np.full((B, most), -1, dtype=np.int32)
            for b, p in enumerate(paths):
                acc[b, :len(p)] = p
            st.update(accepted=_dev(acc), n_accepted=_dev(np.array([len(p) for p in paths], dtype=np.int32)),
                      cached_out=torch.empty(B, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2607_19547_amd import binding as cs
        geo = cs.Geo(L, c["q_heads"], H, D, _sections(c), c["dtype"], [0, P], rope_base=BASE)
        batch = cs.Batch(st["cached_len"], st["row_start"], st["table"], st["slot"], st["coords"], st["mask"],
                         max_rows=c["new"])
        st.update(cs=cs, geo=geo, batch=batch)
        if c["op"] == "plan":
            st["plan"] = cs.PagePlan(st["new_len"], st["n_blocks"], st["n_blocks_out"], st["free"], st["free_head"],
                                     st["free_head_out"], st["status"], parent=st["parent"],
                                     coord_base=st["coord_base"])
        else:
            st["pool"] = cs.PagePool(geo, st["kp"], st["vp"])
        if c["op"] == "attend":
            st["ws"] = torch.empty(max(1, cs.tree_attend_paged_workspace(geo, batch)), dtype=torch.uint8,
                                   device="cuda")
    return st


def _theta(c):
    i = torch.arange(c["dim"] // 2, dtype=torch.float64, device="cuda")
    return BASE ** (-2.0 * i / c["dim"])


# ------------------------------------------------------------------ run
def run(st):
    c = st["c"]
    return (_own if own else _plain)[c["op"]](st)


def _own_plan(st):
    st["cs"].batch_plan_pages(st["geo"], st["n_pages"], st["batch"], st["plan"])
    return _plan_out(st)


def _own_append(st):
    st["cs"].qk_norm_rope_append(st["geo"], st["pool"], st["layer"], st["batch"], st["q"], st["k"], st["v"],
                                 st["q_out"], st["wq"], st["wk"], EPS)
    return dict(q=st["q_out"], k=st["kp"], v=st["vp"])


def _own_attend(st):
    st["cs"].tree_attend_paged(st["geo"], st["pool"], st["layer"], st["batch"], st["q"], st["out"], st["lse"],
                               st["ws"])
    return dict(out=st["out"], lse=st["lse"])


def _own_commit(st):
    st["cs"].tree_commit_paged(st["geo"], st["pool"], 0, st["c"]["layers"], st["batch"], st["accepted"],
                               st["n_accepted"], st["cached_out"])
    return dict(k=st["kp"], v=st["vp"], cached=st["cached_out"])


def _plan_out(st):
    o = dict(row_start=st["row_start"], slot=st["slot"], coords=st["coords"], table=st["table"],
             n_blocks=st["n_blocks_out"], free_head=st["free_head_out"], status=st["status"])
    if st["mask"] is not None:
        o["mask"] = st["mask"]
    return o


def _plain_plan(st):
    c, P = st["c"], st["c"]["page"]
    cached, new, held = (st[k].long() for k in ("cached_len", "new_len", "n_blocks"))
    need = (cached + new + P - 1) // P
    grow = (need - held).clamp(min=0)
    first = st["free_head"].long() + torch.cumsum(grow, 0) - grow
    st["row_start"][0] = 0
    st["row_start"][1:] = torch.cumsum(new, 0)
    start = st["row_start"].long()
    col = torch.arange(st["table"].shape[1], device="cuda")[None, :]
    take = (col >= held[:, None]) & (col < (held + grow)[:, None])
    at = (first[:, None] + col - held[:, None]).clamp(0, st["free"].numel() - 1)
    st["table"].copy_(torch.where(take, st["free"][at], st["table"]))
    end = st["free_head"].long() + grow.sum()
    st["status"].bitwise_or_((need > st["table"].shape[1]).any().int() * 2 + (end > st["free"].numel()).int() * 4)
    st["n_blocks_out"].copy_(held + grow)
    st["free_head_out"].copy_(end)
    r = torch.arange(st["n_rows"], device="cuda")
    req = torch.searchsorted(start[1:], r, right=True)
    i = r - start[req]
    pos = cached[req] + i
    st["slot"].copy_(st["table"][req, pos // P].long() * P + pos % P)
    depth = i
    if st["mask"] is not None:
        par = st["parent"].long()
        up = torch.where(par >= 0, start[req] + par, -1)
        words = torch.arange(st["mask"].shape[1], device="cuda")[None, :]
        mask = torch.where(i[:, None] // 64 == words, torch.ones_like(words) << (i % 64)[:, None], 0)
        for _ in range(max(1, math.ceil(math.log2(c["new"] + 1)))):  # pointer doubling
            on = up >= 0
            mask = mask | torch.where(on[:, None], mask[up.clamp(min=0)], 0)
            up = torch.where(on, up[up.clamp(min=0)], -1)
        st["mask"].copy_(mask)
        depth = torch.zeros_like(i)
        for k in range(64):
            depth += ((mask >> k) & 1).sum(1)
        depth -= 1
    st["coords"].copy_((st["coord_base"].long()[req] + depth)[:, None].expand(-1, 3))
    return _plan_out(st)


def _axis(c):
    s = _sections(c)
    return torch.repeat_interleave(torch.arange(3), torch.tensor(s)).cuda()


def _plain_append(st):
    c, P = st["c"], st["c"]["page"]
    half = c["dim"] // 2
    a = st["coords"].double()[:, st.setdefault("axis", _axis(c))] * st["theta"]
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]

    def turned(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        u, v = x[..., :half], x[..., half:]
        return torch.cat([u * cos - v * sin, u * sin + v * cos], -1).to(_dtype(c))

    st["q_out"].copy_(turned(st["q"], st["wq"]))
    page, off = st["slot"].long() // P, st["slot"].long() % P
    st["kp"][:, st["layer"]][page, :, off] = turned(st["k"], st["wk"])
    st["vp"][:, st["layer"]][page, :, off] = st["v"]
    return dict(q=st["q_out"], k=st["kp"], v=st["vp"])


def _plain_attend(st):
    c = st["c"]
    cached, new = _lengths(c)
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    r0 = 0
    for b in range(c["requests"]):
        n, T = int(new[b]), int(cached[b] + new[b])
        pages = st["table"][b, :-(-T // c["page"])].long()
        k, v = (st[x][:, st["layer"]][pages].float().transpose(0, 1).reshape(H, -1, D)[:, :T] for x in ("kp", "vp"))
        q = st["q"][r0:r0 + n].float().view(n, H, G, D).permute(1, 0, 2, 3).reshape(H, n * G, D)
        s = (q @ k.transpose(1, 2).contiguous()).view(H, n, G, T) * (1.0 / math.sqrt(D))
        w = torch.arange(n, device="cuda")
        if st["mask"] is None:
            see = w[None, :] <= w[:, None]
        else:
            see = (st["mask"][r0:r0 + n][:, w // 64] >> (w % 64)[None, :]) & 1 != 0
        tail = s[..., T - n:]
        tail.masked_fill_(~see[None, :, None, :], -math.inf)
        m = s.amax(-1, keepdim=True)
        s.sub_(m).exp_()
        l = s.sum(-1, keepdim=True)
        o = (s.view(H, n * G, T) @ v).view(H, n, G, D) / l
        st["out"][r0:r0 + n] = o.permute(1, 0, 2, 3).reshape(n, H * G, D).to(_dtype(c))
        st["lse"][r0:r0 + n] = (m + torch.log(l))[..., 0].permute(1, 0, 2).reshape(n, H * G)
        r0 += n
    return dict(out=st["out"], lse=st["lse"])


def _plain_commit(st):
    c, P = st["c"], st["c"]["page"]
    acc = st["accepted"].long()
    i = torch.arange(acc.shape[1], device="cuda")[None, :].expand_as(acc)
    on = i < st["n_accepted"][:, None]
    cached = st["cached_len"].long()[:, None]
    # a row that is not accepted, and the first of each path, moves onto itself
    src, dst = cached + torch.where(on, acc, 0), cached + torch.where(on, i, 0)
    ps, pd = (torch.gather(st["table"].long(), 1, x // P) for x in (src, dst))
    for x in ("kp", "vp"):
        st[x][pd, :, :, dst % P] = st[x][ps, :, :, src % P]
    st["cached_out"].copy_(st["cached_len"] + st["n_accepted"])
    return dict(k=st["kp"], v=st["vp"], cached=st["cached_out"])


_plain = dict(plan=_plain_plan, append=_plain_append, attend=_plain_attend, commit=_plain_commit)
_own = dict(plan=_own_plan, append=_own_append, attend=_own_attend, commit=_own_commit)


# ------------------------------------------------------------------ work
def work(case):
    """Every input read once, every output written once, nothing else."""
    c = case
    cached, new = _lengths(c)
    e = 2 if c["dtype"] == "bf16" else 4
    B, rows, D = c["requests"], int(new.sum()), c["dim"]
    if c["op"] == "plan":
        grow = -(-(cached + new) // c["page"]) - -(-cached // c["page"])
        per_row = 16 + ((4 + 8 * _mask_words(c)) if c["tree"] else 0)
        return {"bytes": int(24 * B + 8 * int(grow.sum()) + per_row * rows), "flops": 10 * rows}
    if c["op"] == "append":
        heads = c["q_heads"] + 2 * c["kv_heads"]
        return {"bytes": rows * (2 * heads * D * e + 16), "flops": rows * (heads - c["kv_heads"]) * D * 8}
    if c["op"] == "commit":
        moved = 3 * B  # the rows of a path that move, about
        return {"bytes": moved * c["layers"] * c["kv_heads"] * D * e * 4, "flops": 0}
    kv = int((cached + new).sum()) * c["kv_heads"] * D * e * 2
    io = rows * c["q_heads"] * (D * e * 2 + 4)
    seen = float((new * cached).sum() + ((new * (new + 1) // 2).sum() if not c["tree"] else (new * 8).sum()))
    return {"bytes": kv + io, "flops": int(4 * D * c["q_heads"] * seen)}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    st = prepare(case, seed)
    return dict(plan=_exact_plan, append=_exact_append, attend=_exact_attend, commit=_exact_commit)[case["op"]](st)


def _exact_plan(st):
    """Whole numbers, request by request on the host."""
    c, P = st["c"], st["c"]["page"]
    cached, new, held, free = (st[k].tolist() for k in ("cached_len", "new_len", "n_blocks", "free"))
    head = int(st["free_head"])
    table, parent, base = st["table"].tolist(), None, st["coord_base"].tolist()
    if st["mask"] is not None:
        parent = st["parent"].tolist()
    start, slot, coords, mask, blocks = [0], [], [], [], []
    for b in range(c["requests"]):
        need = -(-(cached[b] + new[b]) // P)
        for x in range(held[b], need):
            table[b][x] = free[head]
            head += 1
        blocks.append(max(held[b], need))
        seen = []
        for i in range(new[b]):
            p = i - 1 if parent is None else parent[start[b] + i]
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            depth = bin(seen[i]).count("1") - 1
            slot.append(table[b][(cached[b] + i) // P] * P + (cached[b] + i) % P)
            coords.append([base[b] + depth] * 3)
            if parent is not None:
                word = [(seen[i] >> 64 * w) & (1 << 64) - 1 for w in range(_mask_words(c))]
                mask.append([w - (1 << 64) if w >> 63 else w for w in word])
        start.append(start[b] + new[b])
    out = dict(row_start=start, slot=slot, coords=coords, table=table, n_blocks=blocks, free_head=[head], status=[0])
    out = {k: np.array(v, dtype=np.int32) for k, v in out.items()}
    if parent is not None:
        out["mask"] = np.array(mask, dtype=np.int64)
    return {k: torch.from_numpy(v) for k, v in out.items()}


def _exact_append(st):
    """Rotation as a product of complex numbers."""
    c, P, half = st["c"], st["c"]["page"], st["c"]["dim"] // 2
    axis = [0] * _sections(c)[0] + [1] * _sections(c)[1] + [2] * _sections(c)[2]
    angle = torch.stack([st["coords"][:, axis[d]].double() * BASE ** (-2.0 * d / c["dim"]) for d in range(half)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)

    def head(x, w):
        x = x.double()
        x = x / (x.pow(2).sum(-1) / c["dim"] + EPS).sqrt()[..., None] * w.double()
        z = torch.complex(x[:, :half], x[:, half:]) * turn
        return torch.cat([z.real, z.imag], 1)

    q = torch.stack([head(st["q"][:, h], st["wq"]) for h in range(c["q_heads"])], 1)
    k, v = st["kp"].double(), st["vp"].double()
    page, off = torch.div(st["slot"], P, rounding_mode="floor").long(), (st["slot"] % P).long()
    for h in range(c["kv_heads"]):
        k[page, st["layer"], h, off] = head(st["k"][:, h], st["wk"])
        v[page, st["layer"], h, off] = st["v"][:, h].double()
    return dict(q=q, k=k, v=v)


def _exact_attend(st):
    """One query head of one request at a time, keys gathered token by token."""
    c, P, D = st["c"], st["c"]["page"], st["c"]["dim"]
    G = c["q_heads"] // c["kv_heads"]
    out = torch.zeros((st["n_rows"], c["q_heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((st["n_rows"], c["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    start = st["row_start"].tolist()
    for b, past in enumerate(st["cached_len"].tolist()):
        lo, hi = start[b], start[b + 1]
        j = torch.arange(past + hi - lo, device="cuda")
        page, off = st["table"][b][j // P].long(), j % P
        allowed = torch.ones((hi - lo, past + hi - lo), dtype=torch.bool, device="cuda")
        for w in range(hi - lo):
            col = (torch.arange(hi - lo, device="cuda") >= w if st["mask"] is None
                   else (st["mask"][lo:hi, w // 64] >> (w % 64)) & 1 == 1)
            allowed[:, past + w] = col
        for h in range(c["kv_heads"]):
            k = st["kp"][page, st["layer"], h, off].double()
            v = st["vp"][page, st["layer"], h, off].double()
            for x in range(G):
                s = st["q"][lo:hi, h * G + x].double() @ k.t().contiguous() / math.sqrt(D)
                s = s.masked_fill(~allowed, -math.inf)
                z = torch.logsumexp(s, 1)
                out[lo:hi, h * G + x] = torch.exp(s - z[:, None]) @ v
                lse[lo:hi, h * G + x] = z
    return dict(out=out, lse=lse)


def _exact_commit(st):
    """Row by row; the sources of a path are read before any of them is overwritten."""
    P = st["c"]["page"]
    table, past = st["table"].tolist(), st["cached_len"].tolist()
    count = st["n_accepted"].tolist()
    k, v = st["kp"].clone(), st["vp"].clone()
    for b, path in enumerate(st["accepted"].tolist()):
        for i, j in enumerate(path[:count[b]]):
            a, z = past[b] + j, past[b] + i
            for new, old in ((k, st["kp"]), (v, st["vp"])):
                new[table[b][z // P], :, :, z % P] = old[table[b][a // P], :, :, a % P]
    return dict(k=k, v=v, cached=torch.tensor([p + n for p, n in zip(past, count)], dtype=torch.int32))
