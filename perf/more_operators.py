"""Memories held in 4 bits, and attention over a span of them, as measurable cases.

A composed memory that is done with being repaired can be kept in 4 bits: its
full pages go from the pool into a packed pool (2.1 bytes for 4 elements), and
requests are answered from there, their newer tokens in ordinary pages behind.
`op` is one of

  store    pages packed into 4 bits and written back, as the values they then
           stand for
  restore  packed pages back into pool pages, the keys turned by each page's
           offset on the three axes
  attend   attention of a step's rows over packed pages and, behind them,
           ordinary ones; where `window` is not 0, of the tokens that a row sees
           only the first `sinks` and the last `window` count

A value is an element of e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives)
times a power of two that 32 of them share: keys along a token's row, values
along 32 tokens of a channel.  With amax the block's largest magnitude the power
2^e is the least for which amax <= 7 x 2^e, e from -125 to 125; elements are
rounded to nearest, ties to the even code, and saturate at 6.  A packed page is
[L][H_kv] planes, a plane the key codes [P][D/2] (even element in the low half of a
byte), the key scales [P/32][D/32][32] (e + 127), the value codes [P/8][D][4]
(byte w: tokens 2 w and 2 w + 1 of eight) and the value scales [P/32][D].

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
QWEN = dict(q_heads=16, kv_heads=2, dim=128, dtype="bf16")


def _pages(op, **kw):
    c = dict(op=op, pages=1, page=64, layers=36)
    c.update(QWEN)
    c.update(kw)
    return c


def _attend(**kw):
    """packed: tokens in 4 bits (whole pages); recent: cached tokens in ordinary pages behind them."""
    c = dict(op="attend", requests=1, packed=1024, recent=17, new=1, tree=False, page=64, layers=2, ragged=False,
             sinks=0, window=0)
    c.update(QWEN)
    c.update(kw)
    return c


def listed():
    return [
        # A page that an answer has just filled: latency.
        dict(_pages("store", pages=1), name="store-page"),
        # A repaired memory of 8,192 tokens, all 36 layers.
        dict(_pages("store", pages=128), name="store-8k"),
        # Float32, as in fidelity runs, heads of another size, odd counts.
        dict(_pages("store", pages=37, page=96, layers=7, q_heads=10, kv_heads=5, dim=64, dtype="f32"), name="store-f32"),
        # One page moved to another place on the timeline.
        dict(_pages("restore", pages=1), name="restore-page"),
        # A stored memory of 16,384 tokens composed anew: every page moved.
        dict(_pages("restore", pages=256), name="restore-16k"),
        # One answer's next token over a short video's memory.
        dict(_attend(packed=8192, recent=18, new=1), name="decode-8k"),
        # A full server: answers over memories of very different lengths.
        dict(_attend(requests=64, packed=32768, recent=391, new=1, ragged=True), name="decode-64"),
        # A tree of drafted tokens over a long video's memory.
        dict(_attend(packed=65408, recent=101, new=61, tree=True, page=128), name="tree-65k"),
        # Float32: a few small trees over short memories.
        dict(_attend(requests=4, packed=4032, recent=65, new=17, tree=True, ragged=True, dtype="f32", page=96),
             name="tree-4k-f32"),
        # Two questions of a few hundred tokens over long memories: the most
        # arithmetic of all.
        dict(_attend(requests=2, packed=32768, recent=0, new=389), name="question-32k"),
        # Streams that have run for long: the first frame's tokens and the last
        # 4,096 are seen of memories of up to 65,536.
        dict(_attend(requests=48, packed=65536, recent=97, new=1, ragged=True, sinks=196, window=4096),
             name="window-decode"),
        # The next clip of a stream, prefilled behind ordinary pages.
        dict(_attend(packed=0, recent=6001, new=1999, sinks=4, window=1024), name="window-clip"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(16, 2), (16, 2), (28, 4), (40, 8), (10, 10), (12, 1), (4, 2)]


def draw(rng):
    op = rng.choice(["store", "restore", "attend", "attend", "attend"])
    hq, hkv = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([128, 128, 128, 64, 96, 32] if dtype == "bf16" else [128, 64, 32])
    page = rng.choice([32, 64, 64, 96, 128, 256])
    size = 2 if dtype == "bf16" else 4
    kw = dict(q_heads=hq, kv_heads=hkv, dim=dim, dtype=dtype, page=page)
    if op != "attend":
        layers = rng.choice([1, 7, 28, 36])
        most = 300_000_000 // (2 * layers * hkv * page * dim * size)  # pages of the largest listed case's bytes
        return _pages(op, **dict(kw, layers=layers, pages=_log_int(rng, 1, max(2, most))))
    kw["ragged"] = rng.random() < 0.7
    shape = rng.choice(["decode", "decode", "tree", "question"])
    requests = _log_int(rng, 1, 64)
    window = rng.choice([0, 0, _log_int(rng, 1, 8192)])
    sinks = rng.choice([0, 4, _log_int(rng, 1, 512)]) if window else 0
    most = max(page, 180_000_000 // (hkv * dim) // requests)  # tokens a request may have at most
    packed = _log_int(rng, 1, min(65536, most)) // page * page
    recent = _log_int(rng, 1, 1000)
    if window and rng.random() < 0.4:  # ordinary pages alone
        packed, recent = 0, _log_int(rng, 1, min(16384, max(page, most // 4)))
    kw.update(requests=requests, packed=packed, recent=recent, sinks=sinks, window=window)
    if shape == "decode":
        return _attend(**dict(kw, new=1))
    # rows so that the products stay below the largest listed case's
    # (float32: a sixteenth of it, by the rates of the matrix instructions)
    budget = 2 * 389 * 16 * 128 * 33000 // (1 if dtype == "bf16" else 16)
    rows = max(1, budget // (requests * hq * dim * (packed + recent + 256)))
    if shape == "tree":
        return _attend(**dict(kw, new=min(rows, _log_int(rng, 2, 128)), tree=True))
    return _attend(**dict(kw, new=min(rows, _log_int(rng, 2, 512))))


# ------------------------------------------------------------------ sizes
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _sections(c):
    p = c["dim"] // 2
    s = p // 4
    return s, (p - s) // 2, p - s - (p - s) // 2


def _plane(c):
    """Bytes of a packed plane's four parts."""
    P, D = c["page"], c["dim"]
    return P * D // 2, P * D // 32, P * D // 2, P * D // 32


def _lengths(c):
    """(packed, recent, new) of every request; they depend on the case alone, so
    that a case's work does not vary with the seed.  Ragged: spread from a
    sixteenth of the case's length to all of it."""
    B, P = c["requests"], c["page"]
    g = np.random.Generator(np.random.PCG64(B * 1000003 + c["packed"] * 101 + c["recent"] * 7 + c["new"]))
    packed = np.full(B, c["packed"], dtype=np.int64)
    recent = np.full(B, c["recent"], dtype=np.int64)
    new = np.full(B, c["new"], dtype=np.int64)
    if c["ragged"]:
        if c["packed"]:
            packed = np.exp(g.uniform(math.log(c["packed"] / 16), math.log(c["packed"] + 0.5), B)).astype(np.int64)
            packed[0] = c["packed"]
        if c["recent"]:
            recent = g.integers(0, c["recent"] + 1, B)
            recent[0] = c["recent"]
        if c["new"] > 1:
            new = np.maximum(1, g.integers((c["new"] + 1) // 2, c["new"] + 1, B))
            new[0] = c["new"]
    return packed // P * P, recent, new


def _mask_words(c):
    return max(1, -(-c["new"] // 64))


def _parents(new, g):
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
    return out


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _normal(shape, gen, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    return x.normal_(0.0, std, generator=gen)


# ------------------------------------------------------------------ 4 bits, elementary operations in float32
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _scaled(x):
    """Blocks of 32 along the last axis: codes 0 to 15 and the scales' bytes."""
    x = x.float()
    x = x.reshape(*x.shape[:-1], -1, 32)
    e = ((x.abs().amax(-1).view(torch.int32) + 0x1fffff) >> 23).sub_(2).clamp_(2, 252)
    y = x.abs() / (e << 23).view(torch.float32)[..., None]
    code = (y > 0.25).to(torch.uint8)
    for i, b in enumerate((0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += y > b if i % 2 else y >= b
    code += torch.signbit(x) * 8
    return code, e.to(torch.uint8)


def _rounded(x):
    """The values that the blocks of 32 along the last axis stand for."""
    code, e = _scaled(x)
    table = torch.tensor(VALUES, device="cuda")
    y = table[(code & 7).long()] * (e.int() << 23).view(torch.float32)[..., None]
    return torch.where(code >= 8, -y, y).reshape(x.shape)


def _encode(k, v):
    """k, v [..., P, D] (P and D multiples of 32) as planes of bytes [..., plane]."""
    lead, (P, D) = k.shape[:-2], k.shape[-2:]
    code, e = _scaled(k)
    code = code.reshape(*lead, P, D // 2, 2)
    kc = code[..., 0] | code[..., 1] << 4
    ks = e.reshape(*lead, P // 32, 32, D // 32).transpose(-1, -2)
    code, e = _scaled(v.transpose(-1, -2))  # [..., D, P / 32, 32]
    code = code.reshape(*lead, D, P // 8, 4, 2)
    vc = (code[..., 0] | code[..., 1] << 4).transpose(-2, -3)
    vs = e.transpose(-1, -2)
    return torch.cat([x.reshape(*lead, -1) for x in (kc, ks, vc, vs)], -1)


def _decode(c, planes):
    """Planes of bytes [..., plane] as k, v [..., P, D] in float32."""
    lead, P, D = planes.shape[:-1], c["page"], c["dim"]
    kc, ks, vc, vs = torch.split(planes, _plane(c), -1)
    pair = torch.tensor([[s * x for s in (1.0, -1.0) for x in VALUES]], device="cuda")
    pair = torch.stack([pair.expand(16, 16), pair.t().expand(16, 16)], -1).reshape(256, 2)  # both halves of a byte

    def scale(b):
        return (b.int() << 23).view(torch.float32)

    k = pair[kc.int()].reshape(*lead, P // 32, 32, D // 32, 32)
    k = k * scale(ks).reshape(*lead, P // 32, D // 32, 32).transpose(-1, -2)[..., None]
    v = pair[vc.int()].reshape(*lead, P // 32, 4, D, 8) * scale(vs).reshape(*lead, P // 32, 1, D, 1)
    return k.reshape(*lead, P, D), v.transpose(-1, -2).reshape(*lead, P, D)


def _packed_pool(c, n_pages, gen):
    """A packed pool of normal keys and values, made some pages at a time."""
    out = torch.empty((n_pages, c["layers"], c["kv_heads"], sum(_plane(c))), dtype=torch.uint8, device="cuda")
    some = max(1, 30_000_000 // (c["layers"] * c["kv_heads"] * c["page"] * c["dim"]))
    for i in range(0, n_pages, some):
        shape = (min(some, n_pages - i), c["layers"], c["kv_heads"], c["page"], c["dim"])
        k, v = (_normal(shape, gen, torch.float32) for _ in range(2))
        out[i:i + some] = _encode(k, v)
    return out


# ------------------------------------------------------------------ prepare
def prepare(case, seed):
    c = dict(case)
    g = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    st = _prepare_attend(c, g, gen) if c["op"] == "attend" else _prepare_pages(c, g, gen)
    if own:
        from paper_2607_19547_amd import binding as cs
        geo = cs.Geo(c["layers"], c["q_heads"], c["kv_heads"], c["dim"], _sections(c), c["dtype"], [0, c["page"]],
                     rope_base=BASE)
        st.update(cs=cs, geo=geo, pool=cs.PagePool(geo, st["kp"], st["vp"]),
                  packed=None if st["bits"] is None else cs.PackedPool(geo, st["bits"].view(st["bits"].shape[0], -1)))
        if c["op"] == "store":
            st["restored"] = cs.PagePool(geo, st["k_out"], st["v_out"])
        if c["op"] == "attend":
            st["batch"] = cs.Batch(st["cached_len"], st["row_start"], st["table"], st["slot"], st["coords"], st["mask"],
                                   max_rows=c["new"])
            st["ws"] = torch.empty(max(1, cs.tree_attend_packed_workspace(geo, st["batch"])), dtype=torch.uint8,
                                   device="cuda")
    return st


def _prepare_pages(c, g, gen):
    """A pool with a few pages more than are taken, in no order."""
    n = c["pages"] + 3
    shape = (n, c["layers"], c["kv_heads"], c["page"], c["dim"])
    src, dst = (g.permutation(n)[:c["pages"]].astype(np.int32) for _ in range(2))
    st = dict(c=c, src=_dev(src), dst=_dev(dst))
    if c["op"] == "store":
        st.update(kp=_normal(shape, gen, _dtype(c)), vp=_normal(shape, gen, _dtype(c)),
                  bits=torch.zeros(shape[:3] + (sum(_plane(c)),), dtype=torch.uint8, device="cuda"))
        st.update(k_out=torch.zeros_like(st["kp"]), v_out=torch.zeros_like(st["vp"]))
    else:
        move = np.stack([g.integers(-100_000, 100_000, c["pages"]), g.integers(-32, 32, c["pages"]),
                         g.integers(-32, 32, c["pages"])], 1)
        st.update(bits=_packed_pool(c, n, gen), offsets=_dev(move.astype(np.int32)),
                  kp=torch.zeros(shape, dtype=_dtype(c), device="cuda"),
                  vp=torch.zeros(shape, dtype=_dtype(c), device="cuda"))
    return st


def _prepare_attend(c, g, gen):
    packed, recent, new = _lengths(c)
    B, P, H, D, L = c["requests"], c["page"], c["kv_heads"], c["dim"], c["layers"]
    rows, blocks = int(new.sum()), packed // P
    cached = packed + recent
    need = -(-(cached + new) // P)
    plain = need - blocks
    n_bits, n_pages = int(blocks.sum()) + 2, int(plain.sum()) + 2
    table = np.full((B, int(need.max()) + 2), -1, dtype=np.int32)
    order, order4, at, at4 = g.permutation(n_pages), g.permutation(n_bits), 0, 0
    for b in range(B):
        table[b, :blocks[b]] = order4[at4:at4 + blocks[b]]
        table[b, blocks[b]:need[b]] = order[at:at + plain[b]]
        at4, at = at4 + blocks[b], at + plain[b]
    row_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    req = np.repeat(np.arange(B), new)
    idx = np.arange(rows) - row_start[req]
    pos = cached[req] + idx
    slot = table[req, pos // P].astype(np.int64) * P + pos % P
    st = dict(c=c, n_rows=rows, layer=L - 1, cached_len=_dev(cached.astype(np.int32)), table=_dev(table),
              row_start=_dev(row_start), slot=_dev(slot.astype(np.int32)), mask=None,
              coords=_dev(np.repeat(pos[:, None], 3, axis=1).astype(np.int32)))
    if c["tree"]:
        parent = _parents(new, g)
        bits = np.zeros((rows, _mask_words(c)), dtype=np.uint64)
        for r in range(rows):
            i = int(idx[r])
            if parent[r] >= 0:
                bits[r] = bits[r - i + parent[r]]
            bits[r, i // 64] |= np.uint64(1) << np.uint64(i % 64)
        st["mask"] = _dev(bits.view(np.int64))
    dt = _dtype(c)
    st.update(kp=_normal((n_pages, L, H, P, D), gen, dt), vp=_normal((n_pages, L, H, P, D), gen, dt), bits=None,
              blocks=None)
    if c["packed"]:
        st.update(bits=_packed_pool(c, n_bits, gen), blocks=_dev(blocks.astype(np.int32)))
    st["q"] = _normal((rows, c["q_heads"], D), gen, dt, 1.5)
    st["out"] = torch.empty_like(st["q"])
    st["lse"] = torch.empty((rows, c["q_heads"]), dtype=torch.float32, device="cuda")
    return st


# ------------------------------------------------------------------ run
def run(st):
    return (_own if own else _plain)[st["c"]["op"]](st)


def _own_store(st):
    cs, L = st["cs"], st["c"]["layers"]
    cs.pack_pages(st["geo"], st["pool"], st["packed"], 0, L, st["src"], st["dst"])
    cs.unpack_rebase_pages(st["geo"], st["packed"], st["restored"], 0, L, st["dst"], st["dst"])
    return dict(k=st["k_out"], v=st["v_out"])


def _own_restore(st):
    st["cs"].unpack_rebase_pages(st["geo"], st["packed"], st["pool"], 0, st["c"]["layers"], st["src"], st["dst"],
                                 st["offsets"])
    return dict(k=st["kp"], v=st["vp"])


def _own_attend(st):
    st["cs"].tree_attend_packed(st["geo"], st["pool"], st["packed"], st["layer"], st["batch"], st["blocks"], st["q"],
                                st["out"], st["lse"], st["ws"], sinks=st["c"]["sinks"], window=st["c"]["window"])
    return dict(out=st["out"], lse=st["lse"])


def _plain_store(st):
    src, dst = st["src"].long(), st["dst"].long()
    st["k_out"][dst] = _rounded(st["kp"][src]).to(_dtype(st["c"]))
    st["v_out"][dst] = _rounded(st["vp"][src].transpose(-1, -2)).transpose(-1, -2).to(_dtype(st["c"]))
    return dict(k=st["k_out"], v=st["v_out"])


def _plain_restore(st):
    c, half = st["c"], st["c"]["dim"] // 2
    k, v = _decode(c, st["bits"][st["src"].long()])
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(_sections(c))).cuda()
    theta = BASE ** (-2.0 * torch.arange(half, dtype=torch.float64, device="cuda") / c["dim"])
    a = st["offsets"].double()[:, axis] * theta
    cos, sin = (x.float()[:, None, None, None] for x in (torch.cos(a), torch.sin(a)))
    x, y = k[..., :half], k[..., half:]
    dst = st["dst"].long()
    st["kp"][dst] = torch.cat([x * cos - y * sin, x * sin + y * cos], -1).to(_dtype(c))
    st["vp"][dst] = v.to(_dtype(c))
    return dict(k=st["kp"], v=st["vp"])


def _plain_attend(st):
    c, P = st["c"], st["c"]["page"]
    packed, recent, new = _lengths(c)
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    r0 = 0
    for b in range(c["requests"]):
        n, past = int(new[b]), int(packed[b] + recent[b])
        T, blocks = past + n, int(packed[b]) // P
        pages = st["table"][b, blocks:-(-T // P)].long()
        k, v = (st[x][:, st["layer"]][pages].float() for x in ("kp", "vp"))  # [pages, H, P, D]
        if blocks:
            k4, v4 = _decode(c, st["bits"][:, st["layer"]][st["table"][b, :blocks].long()])
            k, v = torch.cat([k4, k]), torch.cat([v4, v])
        k, v = (x.transpose(0, 1).reshape(H, -1, D)[:, :T] for x in (k, v))
        q = st["q"][r0:r0 + n].float().view(n, H, G, D).permute(1, 0, 2, 3).reshape(H, n * G, D)
        s = (q @ k.transpose(1, 2).contiguous()).view(H, n, G, T) * (1.0 / math.sqrt(D))
        w = torch.arange(n, device="cuda")
        if st["mask"] is None:
            see = w[None, :] <= w[:, None]
        else:
            see = (st["mask"][r0:r0 + n][:, w // 64] >> (w % 64)[None, :]) & 1 != 0
        s[..., past:].masked_fill_(~see[None, :, None, :], -math.inf)
        if c["window"]:
            before = torch.cat([torch.arange(past, device="cuda").expand(n, past), past + torch.cumsum(see, 1) - 1], 1)
            hidden = (before >= c["sinks"]) & (before < past + see.sum(1, keepdim=True) - c["window"])
            s.masked_fill_(hidden[None, :, None, :], -math.inf)
        m = s.amax(-1, keepdim=True)
        s.sub_(m).exp_()
        l = s.sum(-1, keepdim=True)
        o = (s.view(H, n * G, T) @ v).view(H, n, G, D) / l
        st["out"][r0:r0 + n] = o.permute(1, 0, 2, 3).reshape(n, H * G, D).to(_dtype(c))
        st["lse"][r0:r0 + n] = (m + torch.log(l))[..., 0].permute(1, 0, 2).reshape(n, H * G)
        r0 += n
    return dict(out=st["out"], lse=st["lse"])


_plain = dict(store=_plain_store, restore=_plain_restore, attend=_plain_attend)
_own = dict(store=_own_store, restore=_own_restore, attend=_own_attend)


# ------------------------------------------------------------------ work
def work(case):
    """Every input read once, every output written once, nothing else; tokens that no row sees are not read."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    H, D = c["kv_heads"], c["dim"]
    if c["op"] != "attend":
        n = c["pages"] * c["layers"] * H * c["page"] * D * 2  # elements
        if c["op"] == "store":
            return {"bytes": n * 2 * e + n * 17 // 32, "flops": n * 4}
        return {"bytes": n * e + n * 17 // 32, "flops": n * 4}
    packed, recent, new = _lengths(c)
    cached, rows = packed + recent, int(new.sum())
    own_rows = new * 8 if c["tree"] else new * (new + 1) // 2  # of a request's new rows, seen by one or another
    read4, read, seen = float(packed.sum()), float((recent + new).sum()), float((new * cached + own_rows).sum())
    if c["window"]:
        # tokens [0, sinks) and, of chains, from the first row's window on
        first = np.maximum(cached + 1 - c["window"], 0)
        lo = np.minimum(c["sinks"], first)
        read4 = float((np.minimum(packed, lo) + np.maximum(packed - first, 0)).sum())
        read = float((lo - np.minimum(packed, lo) + cached + new - np.maximum(first, packed)).sum())
        each = np.minimum(cached + own_rows / new, c["window"] + c["sinks"])
        seen = float((new * each).sum())
    kv = H * D * 2 * (read * e + read4 * 17 / 32)
    io = rows * c["q_heads"] * (D * e * 2 + 4)
    return {"bytes": int(kv + io), "flops": int(4 * D * c["q_heads"] * seen)}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    st = prepare(case, seed)
    return dict(store=_exact_store, restore=_exact_restore, attend=_exact_attend)[case["op"]](st)


def _exact_blocks(x):
    """Blocks of 32 along the last axis, rounded in float64: steps of 0.5 below 2, of 1 below 4, of 2 above."""
    x = x.double().unflatten(-1, (-1, 32))
    mant, e = torch.frexp(x.abs().amax(-1, keepdim=True))  # amax = mant 2^e, 0.5 <= mant < 1
    e = torch.where(mant > 0.875, e - 2, e - 3).clamp(-125, 125)
    y = torch.ldexp(x.abs(), -e)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    y = torch.minimum(torch.round(y / step) * step, torch.full_like(y, 6.0))
    return torch.copysign(torch.ldexp(y, e), x).flatten(-2)


def _exact_store(st):
    k, v = torch.zeros_like(st["k_out"]).double(), torch.zeros_like(st["v_out"]).double()
    for a, z in zip(st["src"].tolist(), st["dst"].tolist()):
        k[z] = _exact_blocks(st["kp"][a])
        v[z] = _exact_blocks(st["vp"][a].transpose(-1, -2).contiguous()).transpose(-1, -2)
    return dict(k=k, v=v)


def _exact_nibbles(b, odd):
    """e2m1 from its bits: sign, two of the exponent, one of the mantissa."""
    x = (b >> 4 if odd else b & 15).long()
    expo, mant = x >> 1 & 3, x & 1
    y = torch.where(expo == 0, 0.5 * mant, (1 + 0.5 * mant) * torch.pow(2.0, expo.double() - 1)).double()
    return torch.where(x > 7, -y, y)


def _exact_plane(c, plane):
    """One plane (or several) of bytes as k, v [..., P, D] in float64, even and odd halves of the bytes apart."""
    P, D = c["page"], c["dim"]
    end = np.cumsum(_plane(c))
    kb, ks, vb, vs = (plane[..., a:z].long() for a, z in zip([0, *end[:-1]], end))
    lead = plane.shape[:-1]
    k = torch.empty(lead + (P, D), dtype=torch.float64, device="cuda")
    v = torch.empty_like(k)
    tok = torch.arange(P, device="cuda")
    kb, vb = kb.view(lead + (P, D // 2)), vb.view(lead + (P // 8, D, 4))
    for odd in (0, 1):
        k[..., odd::2] = _exact_nibbles(kb, odd)
        for w in range(4):
            v[..., 2 * w + odd::8, :] = _exact_nibbles(vb[..., w], odd)
    ks, vs = ks.view(lead + (P // 32, D // 32, 32)), vs.view(lead + (P // 32, D))
    for d in range(D // 32):
        k[..., 32 * d:32 * d + 32] *= torch.pow(2.0, ks[..., tok // 32, d, tok % 32].double() - 127)[..., None]
    v *= torch.pow(2.0, vs[..., tok // 32, :].double() - 127)
    return k, v


def _exact_restore(st):
    """Rotation as a product of complex numbers."""
    c, half = st["c"], st["c"]["dim"] // 2
    axis = [0] * _sections(c)[0] + [1] * _sections(c)[1] + [2] * _sections(c)[2]
    k, v = torch.zeros_like(st["kp"]).double(), torch.zeros_like(st["vp"]).double()
    for a, z, move in zip(st["src"].tolist(), st["dst"].tolist(), st["offsets"].tolist()):
        x, v[z] = _exact_plane(c, st["bits"][a])
        angle = torch.tensor([move[axis[d]] * BASE ** (-2.0 * d / c["dim"]) for d in range(half)], dtype=torch.float64,
                             device="cuda")
        y = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * torch.polar(torch.ones_like(angle),
                                                                                                 angle)
        k[z] = torch.cat([y.real, y.imag], -1)
    return dict(k=k, v=v)


def _exact_attend(st):
    """One query head of one request at a time; a row's tokens are listed, and the ones its window keeps counted off."""
    c, P, D = st["c"], st["c"]["page"], st["c"]["dim"]
    G = c["q_heads"] // c["kv_heads"]
    out = torch.zeros((st["n_rows"], c["q_heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((st["n_rows"], c["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    start = st["row_start"].tolist()
    blocks = [0] * c["requests"] if st["blocks"] is None else st["blocks"].tolist()
    for b, past in enumerate(st["cached_len"].tolist()):
        lo, hi = start[b], start[b + 1]
        n, T = hi - lo, past + hi - lo
        j = torch.arange(blocks[b] * P, T, device="cuda")
        page, off = st["table"][b][j // P].long(), j % P
        allowed = torch.ones((n, T), dtype=torch.bool, device="cuda")
        for w in range(n):
            allowed[:, past + w] = (torch.arange(n, device="cuda") >= w if st["mask"] is None
                                    else (st["mask"][lo:hi, w // 64] >> (w % 64)) & 1 == 1)
        if c["window"]:
            nth = allowed.long().cumsum(1)  # the n-th token that the row sees
            allowed &= (nth <= c["sinks"]) | (nth > allowed.sum(1, keepdim=True) - c["window"])
        for h in range(c["kv_heads"]):
            k = st["kp"][page, st["layer"], h, off].double()
            v = st["vp"][page, st["layer"], h, off].double()
            if blocks[b]:
                k4, v4 = _exact_plane(c, st["bits"][st["table"][b][:blocks[b]].long(), st["layer"], h])
                k, v = torch.cat([k4.flatten(0, 1), k]), torch.cat([v4.flatten(0, 1), v])
            for x in range(G):
                s = st["q"][lo:hi, h * G + x].double() @ k.t().contiguous() / math.sqrt(D)
                s = s.masked_fill(~allowed, -math.inf)
                z = torch.logsumexp(s, 1)
                out[lo:hi, h * G + x] = torch.exp(s - z[:, None]) @ v
                lse[lo:hi, h * G + x] = z
    return dict(out=out, lse=lse)
