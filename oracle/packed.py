"""Float64 oracle of pages held in 4 bits and of attention over them and over windows.

Written from the definitions: an element is the nearest of the sixteen values of
e2m1 times its block's power of two, found by comparing with all of them; a row's
window is counted off the list of the tokens that it sees."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponent(amax):
    """The least e from -125 to 125 with amax <= 7 x 2^e, or 125 where there is none."""
    e = -125
    while e < 125 and amax > 7.0 * 2.0 ** e:
        e += 1
    return e


def block(x):
    """x: 32 values in float64.  (codes 0 to 15, scale byte)."""
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    e = exponent(np.abs(x).max())
    y = np.abs(x) / 2.0 ** e
    d = np.abs(y[:, None] - VALUES)
    near = d == d.min(1, keepdims=True)
    code = np.where(near[:, ::2].any(1), 2 * near[:, ::2].argmax(1), 2 * near[:, 1::2].argmax(1) + 1)
    return (code + 8 * np.signbit(x)).astype(np.uint8), e + 127


def blocks(x):
    """Blocks along the last axis, [..., n]: codes [..., n], scale bytes [..., n / 32]."""
    flat = np.asarray(x, np.float64).reshape(-1, 32)
    out = [block(r) for r in flat]
    return (np.array([c for c, _ in out]).reshape(x.shape),
            np.array([s for _, s in out], np.uint8).reshape(x.shape[:-1] + (x.shape[-1] // 32,)))


def value(code, scale):
    """What codes and (broadcast) scale bytes stand for."""
    s = np.where(scale == 255, np.nan, 2.0 ** (np.minimum(scale, 254).astype(np.float64) - 127))
    y = VALUES[code & 7] * s
    return np.where(code >= 8, -y, y)


def plane_bytes(page, d):
    return page * d * 17 // 16


def encode_plane(k, v):
    """A plane's keys and values [P, D] as its bytes."""
    p, d = k.shape
    kc, ks = blocks(k)
    vc, vs = blocks(np.ascontiguousarray(v.T))
    vc = vc.reshape(d, p // 8, 4, 2).transpose(1, 0, 2, 3)
    return np.concatenate([(kc[:, ::2] | kc[:, 1::2] << 4).reshape(-1),
                           ks.reshape(p // 32, 32, d // 32).transpose(0, 2, 1).reshape(-1),
                           (vc[..., 0] | vc[..., 1] << 4).reshape(-1), vs.T.reshape(-1)]).astype(np.uint8)


def decode_plane(b, p, d):
    """(k, v) [P, D] in float64."""
    n, s = p * d // 2, p * d // 32
    kb, ks, vb, vs = b[:n].reshape(p, d // 2), b[n:n + s], b[n + s:2 * n + s].reshape(p // 8, d, 4), b[2 * n + s:]
    k, v = np.empty((p, d)), np.empty((p, d))
    kc, vc = np.empty((p, d), np.uint8), np.empty((p, d), np.uint8)
    kc[:, ::2], kc[:, 1::2] = kb & 15, kb >> 4
    for w in range(4):
        vc[2 * w::8], vc[2 * w + 1::8] = vb[:, :, w] & 15, vb[:, :, w] >> 4
    ks = ks.reshape(p // 32, d // 32, 32).transpose(0, 2, 1).reshape(p, d // 32)
    k = value(kc, np.repeat(ks, 32, axis=1))
    v = value(vc, np.repeat(vs.reshape(p // 32, d), 32, axis=0))
    return k, v


def decode(pages, layers, hkv, p, d):
    """Packed pages [n, bytes] as (k, v) [n, L, H_kv, P, D] in float64."""
    planes = pages.reshape(-1, plane_bytes(p, d))
    kv = [decode_plane(x, p, d) for x in planes]
    shape = (pages.shape[0], layers, hkv, p, d)
    return np.array([x for x, _ in kv]).reshape(shape), np.array([x for _, x in kv]).reshape(shape)


def encode(k, v):
    """Pages [n, L, H_kv, P, D] as packed pages [n, bytes]."""
    n, layers, hkv, p, d = k.shape
    planes = [encode_plane(a, b) for a, b in zip(k.reshape(-1, p, d), v.reshape(-1, p, d))]
    return np.array(planes, np.uint8).reshape(n, -1)


def visible(cached, mask, n, sinks, window):
    """The tokens that a row sees: the cached ones and the rows of its mask (a python int), of those the first
    `sinks` and the last `window` (window 0: all)."""
    keys = list(range(cached)) + [cached + w for w in range(n) if mask >> w & 1]
    if window and len(keys) > sinks + window:
        keys = keys[:sinks] + keys[len(keys) - window:]
    return keys


def attend(q, k_pool, v_pool, k4, v4, layer, cached, row_start, table, packed_blocks, mask, sinks, window, out, lse,
           spread=None):
    """As oracle.batch.attend, the first packed_blocks[b] pages of a request in the packed pool (decoded: k4, v4)."""
    page, d = k_pool.shape[3:]
    g = q.shape[1] // k_pool.shape[2]
    for b in range(len(cached)):
        lo, hi = row_start[b], row_start[b + 1]
        packed = min(int(packed_blocks[b]), int(cached[b]) // page) if packed_blocks is not None else 0
        for r in range(lo, hi):
            m = (1 << (r - lo + 1)) - 1 if mask is None else mask[r]
            keys = []
            for j in visible(int(cached[b]), m, hi - lo, sinks, window):
                x = j // page
                if x < len(table[b]) and 0 <= table[b][x] < (len(k4) if x < packed else len(k_pool)):
                    keys.append(j)
            if not keys:
                out[r], lse[r] = 0.0, -np.inf
                continue
            x, off = np.array(keys) // page, np.array(keys) % page
            pg, is4 = np.array([table[b][i] for i in x]), x < packed
            for h in range(q.shape[1]):
                kk, vv = np.empty((len(keys), d)), np.empty((len(keys), d))
                kk[~is4], vv[~is4] = (a[pg[~is4], layer, h // g, off[~is4]] for a in (k_pool, v_pool))
                if is4.any():
                    kk[is4], vv[is4] = (a[pg[is4], layer, h // g, off[is4]] for a in (k4, v4))
                qh = np.asarray(q[r, h], np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = kk @ qh / np.sqrt(d)
                    e = np.exp(s - s.max())
                    out[r, h] = e @ vv / e.sum()
                    lse[r, h] = s.max() + np.log(e.sum())
                    if spread is not None:
                        spread[r, h, :d] = e @ np.abs(vv) / e.sum()
                        spread[r, h, d] = (np.abs(kk) @ np.abs(qh)).max() / np.sqrt(d)
                        spread[r, h, d + 1] = len(keys)
