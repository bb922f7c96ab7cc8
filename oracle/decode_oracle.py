"""The decode side from its definitions, in numpy and 64 bits, sequence by sequence: test infrastructure only, sharing
nothing with the library.  A cache is (k, v, pages): pools [pages, heads, page_size, dim] and a table [batch, max_pages]."""
import numpy as np


def _page(pool, table_row, slot):
    """(page, slot in it) of a slot, or None where the page is not in the pool."""
    page = int(table_row[slot // pool.shape[2]])
    return (page, slot % pool.shape[2]) if 0 <= page < pool.shape[0] else None


def visible_slots(pool, table_row, length, most, mask_row=None):
    out = []
    for t in range(max(0, min(int(length), most, table_row.size * pool.shape[2]))):
        if mask_row is not None and not (int(mask_row[t >> 6]) >> (t & 63)) & 1:
            continue
        if _page(pool, table_row, t) is not None:
            out.append(t)
    return out


def attention(k, v, pages, q, lengths, most, scale, mask=None):
    """out, lse, p (a dict per sequence: the visible slots and [q heads, slots]), and what the error bounds need: sum |p v| and,
    per head, the largest scale * sum |q k|."""
    batch, q_heads, dim = q.shape
    group = q_heads // k.shape[1]
    out, lse = np.zeros(q.shape), np.full((batch, q_heads), -np.inf)
    spread, steep = np.zeros(q.shape), np.zeros((batch, q_heads))
    probs = []
    for b in range(batch):
        slots = visible_slots(k, pages[b], lengths[b], most, None if mask is None else mask[b])
        p = np.zeros((q_heads, len(slots)))
        if slots:
            at = np.array([_page(k, pages[b], t) for t in slots])
            for h in range(q_heads):
                kk, vv = (pool[at[:, 0], h // group, at[:, 1]].astype(np.float64) for pool in (k, v))
                s = scale * (kk @ q[b, h].astype(np.float64))
                top = s.max()
                e = np.exp(s - top)
                lse[b, h] = top + np.log(e.sum())
                p[h] = e / e.sum()
                out[b, h] = p[h] @ vv
                spread[b, h] = p[h] @ np.abs(vv)
                steep[b, h] = abs(scale) * (np.abs(kk) @ np.abs(q[b, h].astype(np.float64))).max()
        probs.append((slots, p))
    return out, lse, probs, spread, steep


def append(k, v, pages, lengths, seen, new_k, new_v, counts=None, weights=None, positions=None):
    """In place; returns the new (lengths, seen)."""
    capacity = pages.shape[1] * k.shape[2]
    lengths, seen = np.clip(lengths, 0, capacity), seen.copy()
    for b in range(pages.shape[0]):
        n = new_k.shape[1] if counts is None else min(max(int(counts[b]), 0), new_k.shape[1])
        for t in range(n):
            if lengths[b] >= capacity:
                break
            slot = int(lengths[b])
            at = _page(k, pages[b], slot)
            if at is not None:
                k[at[0], :, at[1]] = new_k[b, t]
                v[at[0], :, at[1]] = new_v[b, t]
            if weights is not None:
                weights[b, :, slot] = 0
            if positions is not None:
                positions[b, :, slot] = seen[b]
            lengths[b] += 1
            seen[b] += 1
    return lengths, seen


def evict(k, v, pages, lengths, seen, weights, positions, budget, recent, most):
    """In place on k, v, weights and positions; returns the new lengths."""
    capacity = pages.shape[1] * k.shape[2]
    out = np.clip(lengths, 0, min(most, capacity))
    for b in range(pages.shape[0]):
        n = int(out[b])
        if n <= budget:
            continue
        out[b] = budget
        for h in range(k.shape[1]):
            def rank(t):
                if positions[b, h, t] >= int(seen[b]) - recent:
                    return (0, 0.0, t)
                w = float(weights[b, h, t])
                return (2, 0.0, t) if w != w else (1, -w, t)
            keep = set(sorted(range(n), key=rank)[:budget])
            holes = [t for t in range(budget) if t not in keep]
            movers = [t for t in range(budget, n) if t in keep]
            assert len(holes) == len(movers)
            for to, frm in zip(holes, movers):
                weights[b, h, to], positions[b, h, to] = weights[b, h, frm], positions[b, h, frm]
                a, z = _page(k, pages[b], to), _page(k, pages[b], frm)
                if a is not None and z is not None:
                    k[a[0], h, a[1]] = k[z[0], h, z[1]]
                    v[a[0], h, a[1]] = v[z[0], h, z[1]]
    return out


def q4_dense(codes, scales, zeros, cols, group):
    """The matrix that codes, scales and zero points stand for, in 64 bits."""
    rows = codes.shape[0]
    w = np.zeros((rows, cols))
    for j in range(cols):
        c = (codes[:, j // 2] >> (4 * (j % 2))) & 15
        g = j // group
        w[:, j] = (c.astype(np.float64) - (8 if zeros is None else zeros[:, g].astype(np.float64))) * scales[:, g].astype(np.float64)
    return w
