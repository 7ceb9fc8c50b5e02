"""Plain 64-bit definitions of the paged KV cache's operators (NumPy, loops over sequences and heads).

Shares no code with the HIP path.  Pages are [n_pages][Hkv][page][D] arrays of float64 (8-bit pages: the codes' values), a table
row names a sequence's pages, lengths are plain integers.
"""
import numpy as np


def rotate(x, pos, inv_freq, interleaved):
    """x [T][heads][D] float64 -> the first 2 len(inv_freq) elements of every head turned by pos * inv_freq."""
    y = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    for t, p in enumerate(pos):
        for i, f in enumerate(np.asarray(inv_freq, dtype=np.float64)):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = np.cos(p * f), np.sin(p * f)
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def norm(x, weight, eps):
    """x [T][heads][D], weight [D] or [heads][D], float64 -> every head divided by the root of its mean square (and eps), times the weight."""
    y = np.empty_like(np.asarray(x, dtype=np.float64))
    weight = np.broadcast_to(np.asarray(weight, dtype=np.float64), y.shape[1:])
    for t in range(y.shape[0]):
        for h in range(y.shape[1]):
            row = np.asarray(x[t, h], dtype=np.float64)
            y[t, h] = row / np.sqrt(np.mean(row * row) + eps) * weight[h]
    return y


def places(table, seq, pos, page, n_pages):
    """(page, row) of every token, None for one that has no place."""
    got = []
    for s, p in zip(seq, pos):
        ok = p >= 0 and 0 <= s < len(table) and p // page < len(table[0]) and 0 <= table[s][p // page] < n_pages
        got.append((int(table[s][p // page]), int(p % page)) if ok else None)
    return got


def span(n, page, window, n_sel, chosen):
    """Token numbers that a query attends to."""
    if chosen is not None:
        return [j for c in chosen for j in range(c * page, min((c + 1) * page, n))]
    return list(range(max(0, n - window) if window else 0, n))


def choose(q, k_min, k_max, n_blocks, n_sel, first, last):
    """Pages for one key/value head: q [G][D], k_min / k_max [n_blocks][D] -> ascending page numbers.

    A page's score is the largest of its heads' sums of q_d k_max_d where q_d is positive and q_d k_min_d elsewhere; sums that are no numbers are
    passed over, and a page without any comes last.  So does one with a dimension that holds no number (k_min +inf, k_max -inf): its sums
    are -inf or no numbers.
    """
    if n_blocks <= n_sel:
        return list(range(n_blocks))
    always = set(range(first)) | set(range(n_blocks - last, n_blocks))
    score = {}
    for p in range(n_blocks):
        if p not in always:
            with np.errstate(invalid="ignore"):
                sums = [float(np.sum(qh * np.where(qh > 0, k_max[p], k_min[p]))) for qh in q]
            score[p] = max([s for s in sums if not np.isnan(s)], default=-np.inf)
    order = sorted(score, key=lambda p: (-score[p], p))
    return sorted(always | set(order[:n_sel - len(always)]))


def attend(q, k, v, table, lens, scale, window=0, chosen=None, k_scale=None, v_scale=None):
    """q [B][Hq][Dk]; k, v pages; chosen[b][hk]: pages to attend to (None: all) -> out [B][Hq][Dv], lse [B][Hq] float64."""
    B, Hq, _ = q.shape
    n_pages, Hkv, page, Dv = v.shape
    G = Hq // Hkv
    out, lse = np.zeros((B, Hq, Dv)), np.full((B, Hq), -np.inf)
    room = table.shape[1] * page
    for b in range(B):
        n = min(max(int(lens[b]), 0), room)
        for hk in range(Hkv):
            at = span(n, page, window, None, None if chosen is None else chosen[b][hk])
            at = [j for j in at if 0 <= table[b][j // page] < n_pages]
            if not at:
                continue
            pg, row = table[b][np.array(at) // page], np.array(at) % page
            keys = k[pg, hk, row] * (1.0 if k_scale is None else float(k_scale[hk]))
            vals = v[pg, hk, row] * (1.0 if v_scale is None else float(v_scale[hk]))
            for h in range(hk * G, (hk + 1) * G):
                z = scale * (keys @ q[b, h])
                m = z.max()
                p = np.exp(z - m)
                out[b, h] = p @ vals / p.sum()
                lse[b, h] = m + np.log(p.sum())
    return out, lse


def attend_shared(q, k, v, table, lens, scale, starts, prefix, k_scale=None, v_scale=None):
    """attend, where the first prefix[g] tokens of those of sequences starts[g] to starts[g + 1] that have as many lie where the row of the first of these says."""
    n_pages, Hkv, page, Dv = v.shape
    (B, Hq, _), G, room = q.shape, q.shape[1] // Hkv, table.shape[1] * page
    out, lse = np.zeros((B, Hq, Dv)), np.full((B, Hq), -np.inf)
    for b in range(B):
        n = min(max(int(lens[b]), 0), room)
        rows = [(b, j) for j in range(n)]
        for g in range(len(prefix)):
            p = min(max(int(prefix[g]), 0), room)
            if starts[g] <= b < starts[g + 1] and n >= p:
                first = next(i for i in range(starts[g], b + 1) if int(lens[i]) >= p)
                rows = [(first if j < p else b, j) for j in range(n)]
        at = [(int(table[r][j // page]), j % page) for r, j in rows]
        at = np.array([(i, r) for i, r in at if 0 <= i < n_pages], dtype=np.int64).reshape(-1, 2)
        if not len(at):
            continue
        for hk in range(Hkv):
            keys = k[at[:, 0], hk, at[:, 1]] * (1.0 if k_scale is None else float(k_scale[hk]))
            vals = v[at[:, 0], hk, at[:, 1]] * (1.0 if v_scale is None else float(v_scale[hk]))
            for h in range(hk * G, (hk + 1) * G):
                z = scale * (keys @ q[b, h])
                w = np.exp(z - z.max())
                out[b, h], lse[b, h] = w @ vals / w.sum(), z.max() + np.log(w.sum())
    return out, lse


def attend_weights(q, k, table, lens, lse, scale, window=0, k_scale=None):
    """What every token is given: [B][Hkv][tokens of the table] sums over a group's heads of exp(scale q.k - lse), 0 where nothing is."""
    n_pages, Hkv, page, _ = k.shape
    B, G, room = q.shape[0], q.shape[1] // Hkv, table.shape[1] * page
    w = np.zeros((B, Hkv, room))
    for b in range(B):
        n = min(max(int(lens[b]), 0), room)
        at = [j for j in span(n, page, window, None, None) if 0 <= table[b][j // page] < n_pages]
        if not at:
            continue
        pg, row = table[b][np.array(at) // page], np.array(at) % page
        for hk in range(Hkv):
            keys = k[pg, hk, row] * (1.0 if k_scale is None else float(k_scale[hk]))
            for h in range(hk * G, (hk + 1) * G):
                w[b, hk, at] += np.exp(scale * (keys @ q[b, h]) - lse[b, h])
    return w


def keep(w, n, n_keep, first, last):
    """Which of n tokens are kept, ascending: the first, the last, and of the others those with the largest w (no number: -inf; ties: the lower)."""
    if n <= n_keep:
        return list(range(n))
    inner = sorted(range(first, n - last), key=lambda j: (-float(w[j]) if w[j] == w[j] else np.inf, j))
    return sorted([*range(first), *inner[:n_keep - first - last], *range(n - last, n)])
