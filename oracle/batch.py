"""Float64 / integer oracle of the batch calls (requests over a pool of pages).

Written from the definitions, request by request; pools are numpy arrays
[n_pages, L, H_kv, P, D] of float64 (or whatever is only moved)."""
import numpy as np


def plan(page, cached, new, held, table, free, head, n_rows, parent=None, base=None, words=0):
    """dict of row_start, table, held, head, slot, coords (depth included) and mask (python ints per row)."""
    table = [list(r) for r in table]
    base = cached if base is None else base
    start, slot, coords, mask, out_held = [0], [], [], [], []
    for b in range(len(cached)):
        need = -(-(int(cached[b]) + int(new[b])) // page)
        for x in range(int(held[b]), need):
            table[b][x] = int(free[head])
            head += 1
        out_held.append(max(int(held[b]), need))
        seen = []
        for i in range(int(new[b])):
            p = i - 1 if parent is None else int(parent[start[b] + i])
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            mask.append(seen[i])
            pos = int(cached[b]) + i
            slot.append(table[b][pos // page] * page + pos % page)
            coords.append([int(base[b]) + bin(seen[i]).count("1") - 1] * 3)
        start.append(start[b] + int(new[b]))
    slot += [-1] * (n_rows - len(slot))
    return dict(row_start=start, table=table, held=out_held, head=head, slot=slot, coords=coords, mask=mask)


def mask_words(mask, words):
    """Masks (python ints) as int64 words, as the device keeps them."""
    full = [[(m >> 64 * w) & ((1 << 64) - 1) for w in range(words)] for m in mask]
    return np.array(full, dtype=np.uint64).reshape(len(mask), words).view(np.int64)


def norm_rope(x, weight, eps, coords, sections, theta):
    """x [n, H, D], weight [D] or None, coords [n, 3], theta [D/2]: the normalised and rotated rows."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    half = x.shape[-1] // 2
    axis = np.repeat(np.arange(3), sections)
    angle = (np.asarray(coords, np.float64)[:, axis] * np.asarray(theta, np.float64))[:, None, :]
    a, b, c, s = x[..., :half], x[..., half:], np.cos(angle), np.sin(angle)
    return np.concatenate([a * c - b * s, a * s + b * c], axis=-1)


def attend(q, k_pool, v_pool, layer, cached, row_start, table, mask, out, lse, spread=None):
    """Writes out [n, H_q, D] and lse [n, H_q] (float64) in place; mask: python ints per row, or None (causal).
    spread [n, H_q, D + 2], where given: sum_j p_j |V_j|, the largest sum_d |q_d K_jd| / sqrt(D), the keys seen."""
    n_pages, _, hkv, page, d = k_pool.shape
    g = q.shape[1] // hkv
    for b in range(len(cached)):
        lo, hi = row_start[b], row_start[b + 1]
        for r in range(lo, hi):
            m = (1 << (r - lo + 1)) - 1 if mask is None else mask[r]
            keys = list(range(int(cached[b]))) + [int(cached[b]) + w for w in range(hi - lo) if m >> w & 1]
            keys = [j for j in keys if j // page < len(table[b]) and 0 <= table[b][j // page] < n_pages]
            if not keys:
                out[r], lse[r] = 0.0, -np.inf
                continue
            pg, off = np.array([table[b][j // page] for j in keys]), np.array(keys) % page
            for h in range(q.shape[1]):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = k_pool[pg, layer, h // g, off].astype(np.float64) @ np.asarray(q[r, h], np.float64) / np.sqrt(d)
                    e = np.exp(s - s.max())
                    out[r, h] = e @ v_pool[pg, layer, h // g, off].astype(np.float64) / e.sum()
                    lse[r, h] = s.max() + np.log(e.sum())
                    if spread is not None:
                        spread[r, h, :d] = e @ np.abs(v_pool[pg, layer, h // g, off].astype(np.float64)) / e.sum()
                        spread[r, h, d] = (np.abs(k_pool[pg, layer, h // g, off]).astype(np.float64)
                                           @ np.abs(np.asarray(q[r, h], np.float64))).max() / np.sqrt(d)
                        spread[r, h, d + 1] = len(keys)


def commit(pools, layers, cached, new, table, accepted, count):
    """Moves the accepted rows in each pool (in place); returns the new cached lengths."""
    page, out = pools[0].shape[3], []
    for b in range(len(cached)):
        moved = 0
        for i in range(min(int(count[b]), len(accepted[b]))):
            j = int(accepted[b][i])
            if j >= new[b] or j <= (int(accepted[b][i - 1]) if i else -1):
                break
            s, t = int(cached[b]) + j, int(cached[b]) + i
            for p in pools:
                p[table[b][t // page], layers[0]:layers[1], :, t % page] = p[table[b][s // page],
                                                                              layers[0]:layers[1], :, s % page]
            moved += 1
        out.append(int(cached[b]) + moved)
    return out
